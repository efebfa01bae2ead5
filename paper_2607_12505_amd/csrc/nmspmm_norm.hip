// The norms around a block with its gate and residual scale, their backward
// pass, and int8 codes of rows with a scale for each.
//
//   u = post(y);  res = alpha r + gate u;  z = pre(res)
//
// A row (token) is read once, stays in the registers of its team of waves, and is
// written once.  A team is as few waves as hold the row in 16 (backward: 8) values
// a lane, so the statistics of up to 1024 (512) channels need no LDS and no
// barrier.  Teams walk over rows with the next row's loads in flight, and keep the
// channel parameters in registers (backward: in LDS).
// Statistics are in binary32, the variance from the centred row (not from the
// difference of two sums, which cancels where the mean is large).
#include <hip/hip_runtime.h>

#include <type_traits>

#include "nmspmm_block.h"
#include "nmspmm_values.h"

namespace nmspmm {
namespace {

typedef unsigned int v2u __attribute__((ext_vector_type(2)));

// A lane's part of a row: CH chunks of VEC consecutive channels, chunk c of
// lane l of the team at channel (c * lanes + l) * VEC.  VEC = 8 needs d % 8 == 0
// and 16-byte aligned rows; any other row goes one channel at a time.
// As loaded: 16-bit values stay two to a register until they are used.
template <class T, int VEC, int CH>
struct Part {
    typename std::conditional<VEC == 8, Raw8<T>, T>::type v[CH];
    __device__ __forceinline__ void get(float (&f)[CH][VEC]) const {
#pragma unroll
        for (int c = 0; c < CH; ++c)
            if constexpr (VEC == 8) {
#pragma unroll
                for (int e = 0; e < 8; ++e) f[c][e] = (float)v[c].v[e];
            } else {
                f[c][0] = (float)v[c];
            }
    }
};

// A row as a buffer: its address is the same for a whole wave and stays in scalar
// registers, a load past its end gives zeros and a store there writes nothing,
// so no lane is masked.  A row of no values reads as zeros.
__device__ __forceinline__ __amdgpu_buffer_rsrc_t row_of(const void *base, int64_t at, int bytes) {
    return __builtin_amdgcn_make_buffer_rsrc((char *)base + at, 0, bytes, 0x00020000);
}
typedef unsigned int v4u __attribute__((ext_vector_type(4)));

template <class T, int VEC, int CH>
__device__ __forceinline__ void load_part(Part<T, VEC, CH> &p, __amdgpu_buffer_rsrc_t row, int at, int step) {
#pragma unroll
    for (int c = 0; c < CH; ++c) {
        const int off = (at + c * step) * (int)sizeof(T);
        if constexpr (VEC == 8 && sizeof(T) == 2) {
            p.v[c] = __builtin_bit_cast(Raw8<T>, __builtin_amdgcn_raw_buffer_load_b128(row, off, 0, 0));
        } else if constexpr (VEC == 8) {
            struct Two {
                v4u lo, hi;
            } two = {__builtin_amdgcn_raw_buffer_load_b128(row, off, 0, 0),
                     __builtin_amdgcn_raw_buffer_load_b128(row, off + 16, 0, 0)};
            p.v[c] = __builtin_bit_cast(Raw8<T>, two);
        } else if constexpr (sizeof(T) == 2) {
            p.v[c] = __builtin_bit_cast(T, (uint16_t)__builtin_amdgcn_raw_buffer_load_b16(row, off, 0, 0));
        } else {
            p.v[c] = __builtin_bit_cast(T, __builtin_amdgcn_raw_buffer_load_b32(row, off, 0, 0));
        }
    }
}
template <class T, int VEC, int CH>
__device__ __forceinline__ void store_part(__amdgpu_buffer_rsrc_t row, const float (&f)[CH][VEC], int at, int step) {
#pragma unroll
    for (int c = 0; c < CH; ++c) {
        const int off = (at + c * step) * (int)sizeof(T);
        if constexpr (VEC == 8) {
            Raw8<T> t;
#pragma unroll
            for (int e = 0; e < 8; ++e) t.v[e] = (T)f[c][e];
            if constexpr (sizeof(T) == 2) {
                __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(v4u, t), row, off, 0, 0);
            } else {
                struct Two {
                    v4u lo, hi;
                };
                const Two two = __builtin_bit_cast(Two, t);
                __builtin_amdgcn_raw_buffer_store_b128(two.lo, row, off, 0, 0);
                __builtin_amdgcn_raw_buffer_store_b128(two.hi, row, off + 16, 0, 0);
            }
        } else if constexpr (sizeof(T) == 2) {
            __builtin_amdgcn_raw_buffer_store_b16(__builtin_bit_cast(uint16_t, (T)f[c][0]), row, off, 0, 0);
        } else {
            __builtin_amdgcn_raw_buffer_store_b32(__builtin_bit_cast(uint32_t, (T)f[c][0]), row, off, 0, 0);
        }
    }
}
// A parameter of the lane's channels, `absent` where there is none and zero past d:
// a lane without channels adds nothing to any sum.
template <int VEC, int CH>
__device__ __forceinline__ void load_param(float (&p)[CH][VEC], const float *row, float absent, int d, int at,
                                           int step) {
    if (row) {
        Part<float, VEC, CH> t;
        load_part(t, row_of(row, 0, d * 4), at, step);
        t.get(p);
    } else {
#pragma unroll
        for (int c = 0; c < CH; ++c)
#pragma unroll
            for (int e = 0; e < VEC; ++e) p[c][e] = at + c * step < d ? absent : 0.f;
    }
}
template <int VEC, int CH>
__device__ __forceinline__ float total(const float (&f)[CH][VEC]) {
    float s = 0.f;
#pragma unroll
    for (int c = 0; c < CH; ++c)
#pragma unroll
        for (int e = 0; e < VEC; ++e) s += f[c][e];
    return s;
}
// Subtracts the mean where the lane holds channels of the row (the others stay
// zero) and returns the sum of squares.
template <int VEC, int CH>
__device__ __forceinline__ float centre(float (&f)[CH][VEC], float mean, int d, int at, int step) {
    float s = 0.f;
#pragma unroll
    for (int c = 0; c < CH; ++c) {
        const float mu = at + c * step < d ? mean : 0.f;
#pragma unroll
        for (int e = 0; e < VEC; ++e) {
            f[c][e] -= mu;
            s = __builtin_fmaf(f[c][e], f[c][e], s);
        }
    }
    return s;
}

constexpr int team_threads(int wpr) { return wpr > 4 ? 64 * wpr : 256; }

// --------------------------------------------------------------- forward
// Bound by memory: 18464 x 1024 bf16 (layer norm before, gate) 27.3 us, 5.5 TB/s of the rows
// read and written, where a copy of 512 MiB reaches 5.3; a gate for each token adds its 4 bytes a
// channel, 37.6 us for 28.8 in a graph.  One token of 1024: 2.4 us.  Past 8192 channels 16 waves of
// 128 registers hold 16 values a lane and spill 83 to 129: 4096 x 12288 bf16 210 us, 1.9 TB/s.
template <class T, int VEC, int CH, int WPR>
__global__ __launch_bounds__(team_threads(WPR)) void k_norm_residual(NormArgs a) {
    constexpr int TEAMS = team_threads(WPR) / 64 / WPR;
    __shared__ float box[TEAMS][2][2][WPR];
    const int team = __builtin_amdgcn_readfirstlane(threadIdx.x / (64 * WPR)), lane = threadIdx.x % (64 * WPR);
    RowReduce<WPR> red{box[team], lane >> 6};
    const int at = lane * VEC, step = 64 * WPR * VEC;
    const float per = 1.f / (float)a.d;
    const int bytes = a.d * (int)sizeof(T);

    float gate[CH][VEC], wq[CH][VEC], bq[CH][VEC], wp[CH][VEC], bp[CH][VEC];
    if (a.groups <= 1) load_param(gate, a.gate, 1.f, a.d, at, step);
    load_param(wp, a.post.weight, 1.f, a.d, at, step);
    load_param(bp, a.post.bias, 0.f, a.d, at, step);
    load_param(wq, a.pre.weight, 1.f, a.d, at, step);
    load_param(bq, a.pre.bias, 0.f, a.d, at, step);

    Part<T, VEC, CH> y = {}, r = {};
    auto fetch = [&](int row) {
        if (row >= a.m) return;
        if (a.y) load_part(y, row_of(a.y, row * a.ldy * (int)sizeof(T), bytes), at, step);
        if (a.r) load_part(r, row_of(a.r, row * a.ldr * (int)sizeof(T), bytes), at, step);
    };
    fetch(blockIdx.x * TEAMS + team);
    for (int row0 = blockIdx.x * TEAMS; row0 < a.m; row0 += gridDim.x * TEAMS) {
        const int row = row0 + team;
        const bool live = row < a.m;
        if (a.groups > 1)
            load_param(gate, a.gate + (int64_t)(live ? row / a.per_group : 0) * a.d, 1.f, a.d, at, step);
        float v[CH][VEC], rf[CH][VEC];
        y.get(v);
        r.get(rf);
        fetch(row + (int)gridDim.x * TEAMS);

        if (a.post.kind != NM_NORM_NONE) {
            const float mean = a.post.kind == NM_NORM_LAYER ? red.sum(total(v)) * per : 0.f;
            const float sq = red.sum(centre(v, mean, a.d, at, step));
            const float scale = 1.f / __builtin_sqrtf(__builtin_fmaf(sq, per, a.post.eps));
#pragma unroll
            for (int c = 0; c < CH; ++c)
#pragma unroll
                for (int e = 0; e < VEC; ++e) v[c][e] = __builtin_fmaf(v[c][e] * scale, wp[c][e], bp[c][e]);
        }
#pragma unroll
        for (int c = 0; c < CH; ++c)
#pragma unroll
            for (int e = 0; e < VEC; ++e)
                v[c][e] = __builtin_fmaf(gate[c][e], v[c][e], a.alpha * rf[c][e]);
        if (a.res && live) store_part<T>(row_of(a.res, (int64_t)row * bytes, bytes), v, at, step);
        if (!a.z && !a.zq) continue;

        // the norm sees the sum before its rounding to T: one rounding for each output
        if (a.pre.kind != NM_NORM_NONE) {
            const float mean = a.pre.kind == NM_NORM_LAYER ? red.sum(total(v)) * per : 0.f;
            const float sq = red.sum(centre(v, mean, a.d, at, step));
            const float scale = 1.f / __builtin_sqrtf(__builtin_fmaf(sq, per, a.pre.eps));
#pragma unroll
            for (int c = 0; c < CH; ++c)
#pragma unroll
                for (int e = 0; e < VEC; ++e) v[c][e] = __builtin_fmaf(v[c][e] * scale, wq[c][e], bq[c][e]);
        }
        if (a.z && live) store_part<T>(row_of(a.z, (int64_t)row * bytes, bytes), v, at, step);
        if (a.zq) {
            float top = 0.f;
#pragma unroll
            for (int c = 0; c < CH; ++c)
#pragma unroll
                for (int e = 0; e < VEC; ++e) top = larger(top, magnitude(v[c][e]));
            const RowScale rs = row_scale(red.largest(top));
            if (live) {
                if (lane == 0) a.zs[row] = rs.scale;
#pragma unroll
                for (int c = 0; c < CH; ++c) {
                    const int ch = at + c * step;
                    if (ch >= a.ldq) continue;     // the codes' rows are padded with zeros
                    int8_t *dst = a.zq + (int64_t)row * a.ldq + ch;
                    int q[VEC];
#pragma unroll
                    for (int e = 0; e < VEC; ++e) q[e] = ch < a.d ? row_code(v[c][e], rs.inv) : 0;
                    if constexpr (VEC == 8)
                        *(v2u *)dst = v2u{pack4(q[0], q[1], q[2], q[3]), pack4(q[4], q[5], q[6], q[7])};
                    else
                        *dst = (int8_t)q[0];
                }
            }
        }
    }
}

// The norms' parameters of the backward pass in LDS, where registers are short:
// as a team's lanes read them, 16 bytes a lane and instruction (VEC = 8: the
// first four channels of every chunk, then the last four).
template <int VEC, int CH, int LANES>
struct SharedParam {
    typedef float v4 __attribute__((ext_vector_type(4)));
    static constexpr int SIZE = LANES * CH * VEC;
    // how many of the three fit beside the rest: past 8192 channels post's bias is read from memory
    static constexpr int FIT = 3 * SIZE * 4 <= 128 * 1024 ? 3 : 2;
    float *at0;
    __device__ void fill(const float *src, float absent, int d) const {
        for (int ch = threadIdx.x; ch < SIZE; ch += blockDim.x) {
            const int to = VEC == 8 ? (ch % 8 / 4) * (LANES * CH * 4) + ch / 8 * 4 + ch % 4 : ch;
            at0[to] = ch < d ? (src ? src[ch] : absent) : 0.f;
        }
    }
    // The first channel of a piece: four floats, or one.
    static __device__ __forceinline__ int channel(int place) {
        return VEC == 8 ? place % (LANES * CH) * 8 + place / (LANES * CH) * 4 : place;
    }
    __device__ __forceinline__ void put(const float (&f)[CH][VEC], int lane) const {
#pragma unroll
        for (int c = 0; c < CH; ++c) {
            if constexpr (VEC == 8) {
                *(v4 *)(at0 + (c * LANES + lane) * 4) = v4{f[c][0], f[c][1], f[c][2], f[c][3]};
                *(v4 *)(at0 + (LANES * CH + c * LANES + lane) * 4) = v4{f[c][4], f[c][5], f[c][6], f[c][7]};
            } else {
                at0[c * LANES + lane] = f[c][0];
            }
        }
    }
    __device__ __forceinline__ void get(float (&f)[CH][VEC], int lane) const {
#pragma unroll
        for (int c = 0; c < CH; ++c) {
            if constexpr (VEC == 8) {
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const v4 t = *(const v4 *)(at0 + h * (LANES * CH * 4) + (c * LANES + lane) * 4);
#pragma unroll
                    for (int e = 0; e < 4; ++e) f[c][4 * h + e] = t[e];
                }
            } else {
                f[c][0] = at0[c * LANES + lane];
            }
        }
    }
};

// --------------------------------------------------------------- backward
// With hat(v) the normalised row and t = dout * weight, a norm's gradient is
//   dv = (t - [mean(t)] - hat * mean(t * hat)) / deviation     ([]: layer norm)
// so: dt = dres + that of pre at res;  dr = alpha dt;  dy = that of post at y,
// of gate * dt.  The statistics are computed again from y and res: the rows are
// in registers, and saved ones would have to be read.
//
// A team takes a run of consecutive rows and sums for its channels what the
// parameters' gradients need; the teams of a workgroup join their sums in LDS,
// the workgroups in k_norm_sums: every addition has its place, so results do not
// change from run to run.  A workgroup is as many teams as a compute unit holds,
// so that few sums are left to join.  A gate that is shared by fewer tokens than all is
// finished, or put aside for k_norm_sums, whenever the team reaches the group's end.
//
// Bound by its own arithmetic: 390 vector instructions for a wave's part of a row
// (18464 x 1024 bf16 with both layer norms 50.7 us, 4.5 TB/s; with 500 of them 55.7, the
// vector units busy 70 % of it).  So two sums share a reduction, and no load or store is
// behind a branch, whose two sides would copy registers.  Short batches are bound by
// what surrounds the rows: with workgroups of 4 waves the 1536 x 1024 sums of three times
// as many workgroups took 25.8 us to leave and add, now 16.7; 12608 x 384 fp16 18.9 us.
//   Registers spill in the forms beside these: 6 to 54 of binary32 rows without a norm after
// (18464 x 1024 111 us, 2048 x 8192 145), 25 to 111 of odd rows past 512 channels with one (4096 x 1021 bf16
// 32 us), 115 and more past 8192 channels (512 x 16384 bf16 93 us, with both norms 236).
// 1 / sqrt(v), within an ulp (the hardware's, which takes no denormals): the root and quotient
// rounded one after the other, as the forward pass has them, took 40 of a row's 500 instructions.
__device__ __forceinline__ float inverse_root(float v) {
    const bool tiny = v < 0x1p-100f;
    return __builtin_amdgcn_rsqf(tiny ? v * 0x1p64f : v) * (tiny ? 0x1p32f : 1.f);
}
// The first row of a run, and the run of a row.
__host__ __device__ constexpr int first_row(int64_t run, int m, int runs) { return (int)(run * m / runs); }
__device__ constexpr int run_of(int64_t row, int m, int runs) { return (int)(((row + 1) * runs - 1) / m); }
// Waves of a SIMD that the register budget is made for.
constexpr int grad_waves(int wpr, int vec, int ch, bool post) {
    return wpr == 16 ? 4 : ch * vec > 8 ? 2 : vec == 8 && !post ? 4 : 3;
}

constexpr int grad_teams(int wpr, int vec, int ch, bool post) {
    if (wpr >= 8 && (post || vec == 1 || wpr == 16)) return 1;
    return 4 * grad_waves(wpr, vec, ch, post) / wpr;
}

// POST: whether there is a norm after the block (its sums are 40 % of the registers).
template <class T, int VEC, int CH, int WPR, bool POST>
__global__ __launch_bounds__(64 * WPR *grad_teams(WPR, VEC, CH, POST))
__attribute__((amdgpu_waves_per_eu(grad_waves(WPR, VEC, CH, POST)))) void k_norm_residual_backward(NormGradArgs a) {
    constexpr int TEAMS = grad_teams(WPR, VEC, CH, POST), LANES = 64 * WPR, SUMS = POST ? 5 : 3;
    __shared__ float box[TEAMS][2][2][WPR];
    // the parameters, then (TEAMS > 1) the sums of every team
    using Shared = SharedParam<VEC, CH, LANES>;
    constexpr int PARAMS = Shared::SIZE * (POST ? Shared::FIT : 1), ALL = TEAMS > 1 ? TEAMS * SUMS * Shared::SIZE : 0;
    __shared__ __attribute__((aligned(16))) float joined[PARAMS > ALL ? PARAMS : ALL];
    const int team = __builtin_amdgcn_readfirstlane(threadIdx.x / LANES), lane = threadIdx.x % LANES;
    RowReduce<WPR> red{box[team], lane >> 6};
    const int at = lane * VEC, step = LANES * VEC;
    const float per = 1.f / (float)a.d;
    const int run = blockIdx.x * TEAMS + team;
    const int first = run < a.runs ? first_row(run, a.m, a.runs) : a.m;
    const int end = run < a.runs ? first_row(run + 1, a.m, a.runs) : a.m;
    const bool layer_q = a.pre.kind == NM_NORM_LAYER, layer_p = a.post.kind == NM_NORM_LAYER;
    const bool has_q = a.pre.kind != NM_NORM_NONE;
    constexpr bool has_p = POST;
    const int bytes = a.d * (int)sizeof(T);

    float gate[CH][VEC] = {};      // of a team without rows too: its zeros must stay zeros
    float s_wq[CH][VEC] = {}, s_bq[CH][VEC] = {}, s_g[CH][VEC] = {}, s_wp[CH][VEC] = {}, s_bp[CH][VEC] = {};
    Part<T, VEC, CH> py = {}, pr = {}, pz = {}, pd = {};
    auto fetch = [&](int row) {
        // a team that is done takes rows of zeros along: they add nothing
        const int n = row < end ? bytes : 0;
        const int64_t r = row < end ? row : 0;
        // (and so does one without the tensor: no branch)
        load_part(py, row_of(a.y, r * a.ldy * (int)sizeof(T), a.y ? n : 0), at, step);
        load_part(pr, row_of(a.res, r * a.ldr * (int)sizeof(T), has_q ? n : 0), at, step);
        load_part(pz, row_of(a.dz, r * a.lddz * (int)sizeof(T), a.dz ? n : 0), at, step);
        load_part(pd, row_of(a.dres, r * a.lddres * (int)sizeof(T), a.dres ? n : 0), at, step);
    };
    fetch(first);
    const Shared lds_wq{joined}, lds_wp{joined + Shared::SIZE}, lds_bp{joined + 2 * Shared::SIZE};
    lds_wq.fill(a.pre.weight, 1.f, a.d);
    if constexpr (POST) {
        lds_wp.fill(a.post.weight, 1.f, a.d);
        if constexpr (Shared::FIT == 3) lds_bp.fill(a.post.bias, 0.f, a.d);
    }
    __syncthreads();
    int group = -1;
    auto group_done = [&]() {
        // a group within this run is finished; one that other runs share is put
        // aside, in place 0 if the run began with it (or within it), else in 1
        const bool whole = group * a.per_group >= first && (group + 1) * a.per_group <= end;
        const float *dst = whole ? a.dgate + (int64_t)group * a.d
                                 : a.gate_parts + ((int64_t)run * 2 + (group == first / a.per_group ? 0 : 1)) * a.d;
        store_part<float>(row_of(dst, 0, a.d * 4), s_g, at, step);
#pragma unroll
        for (int c = 0; c < CH; ++c)
#pragma unroll
            for (int e = 0; e < VEC; ++e) s_g[c][e] = 0.f;
    };
    // every team of the workgroup makes as many turns: the reductions hold barriers
    for (int i = 0; i < a.turns; ++i) {
        const int row = first + i;
        const bool live = row < end;
        if (WPR == 1 && !live) break;
        if (live && (a.groups <= 1 ? group < 0 : row / a.per_group != group)) {
            if (a.groups > 1 && group >= 0 && a.dgate) group_done();
            group = a.groups <= 1 ? 0 : row / a.per_group;
            load_param(gate, a.gate ? a.gate + (int64_t)group * a.d : nullptr, 1.f, a.d, at, step);
        }
        float y[CH][VEC], r[CH][VEC], dz[CH][VEC], dt[CH][VEC];
        py.get(y);
        pr.get(r);
        pz.get(dz);
        pd.get(dt);
        fetch(row + 1);

        float my = has_p ? total(y) : 0.f, mr = total(r);
        if (layer_p || layer_q) red.sum2(my, mr);
        float vy = has_p ? centre(y, layer_p ? my * per : 0.f, a.d, at, step) : 0.f;
        float vr = centre(r, layer_q ? mr * per : 0.f, a.d, at, step);
        red.sum2(vy, vr);
        const float inv_y = has_p ? inverse_root(__builtin_fmaf(vy, per, a.post.eps)) : 1.f;
        if (has_q) {
            const float inv_r = inverse_root(__builtin_fmaf(vr, per, a.pre.eps));
            float st = 0.f, sth = 0.f, wq[CH][VEC];
            lds_wq.get(wq, lane);
#pragma unroll
            for (int c = 0; c < CH; ++c)
#pragma unroll
                for (int e = 0; e < VEC; ++e) {
                    const float hat = r[c][e] * inv_r, g = dz[c][e];
                    s_wq[c][e] = __builtin_fmaf(g, hat, s_wq[c][e]);
                    s_bq[c][e] += g;
                    r[c][e] = hat;
                    dz[c][e] = g * wq[c][e];
                    st += dz[c][e];
                    sth = __builtin_fmaf(dz[c][e], hat, sth);
                }
            red.sum2(st, sth);
            const float mt = layer_q ? st * per : 0.f, mth = sth * per;
#pragma unroll
            for (int c = 0; c < CH; ++c)
#pragma unroll
                for (int e = 0; e < VEC; ++e)
                    dt[c][e] += inv_r * (dz[c][e] - mt - r[c][e] * mth);
        } else {
#pragma unroll
            for (int c = 0; c < CH; ++c)
#pragma unroll
                for (int e = 0; e < VEC; ++e) dt[c][e] += dz[c][e];
        }
        {
            float out[CH][VEC];
#pragma unroll
            for (int c = 0; c < CH; ++c)
#pragma unroll
                for (int e = 0; e < VEC; ++e) out[c][e] = a.alpha * dt[c][e];
            store_part<T>(row_of(a.dr, (int64_t)row * bytes, a.dr && live ? bytes : 0), out, at, step);
        }
        if (!a.y) continue;

        float st = 0.f, sth = 0.f, wp[CH][VEC], bp[CH][VEC];
        if constexpr (POST) {
            lds_wp.get(wp, lane);
            if constexpr (Shared::FIT == 3)
                lds_bp.get(bp, lane);
            else
                load_param(bp, a.post.bias, 0.f, a.d, at, step);
        }
#pragma unroll
        for (int c = 0; c < CH; ++c) {
#pragma unroll
            for (int e = 0; e < VEC; ++e) {
                const float t = dt[c][e];      // past d: times the gate's zero
                if constexpr (POST) {
                    const float hat = y[c][e] * inv_y, g = t * gate[c][e];
                    s_g[c][e] = __builtin_fmaf(t, __builtin_fmaf(hat, wp[c][e], bp[c][e]), s_g[c][e]);
                    s_wp[c][e] = __builtin_fmaf(g, hat, s_wp[c][e]);
                    s_bp[c][e] += g;
                    y[c][e] = hat;
                    dt[c][e] = g * wp[c][e];
                    st += dt[c][e];
                    sth = __builtin_fmaf(dt[c][e], hat, sth);
                } else {
                    s_g[c][e] = __builtin_fmaf(t, y[c][e], s_g[c][e]);
                    dt[c][e] = t * gate[c][e];
                }
            }
        }
        if constexpr (POST) {
            red.sum2(st, sth);
            const float mt = layer_p ? st * per * inv_y : 0.f, mth = sth * per * inv_y;
#pragma unroll
            for (int c = 0; c < CH; ++c)
#pragma unroll
                for (int e = 0; e < VEC; ++e)
                    dt[c][e] = __builtin_fmaf(-y[c][e], mth, __builtin_fmaf(dt[c][e], inv_y, -mt));
        }
        store_part<T>(row_of(a.dy, (int64_t)row * bytes, a.dy && live ? bytes : 0), dt, at, step);
    }
    if (a.groups > 1 && group >= 0 && a.dgate) group_done();

    // this workgroup's sums, in the order gate, pre weight, pre bias, post weight, post bias
    float *const dst[5] = {a.groups <= 1 ? a.dgate : nullptr, a.dpre_weight, a.dpre_bias, a.dpost_weight, a.dpost_bias};
    const int64_t span = (int64_t)gridDim.x * a.d;
    float *parts = a.parts + (int64_t)blockIdx.x * a.d;
    if constexpr (TEAMS == 1) {
        const auto put = [&](int kind, const float (&f)[CH][VEC]) {
            if (dst[kind]) store_part<float>(row_of(parts + kind * span, 0, a.d * 4), f, at, step);
        };
        put(0, s_g);
        put(1, s_wq);
        put(2, s_bq);
        if constexpr (POST) {
            put(3, s_wp);
            put(4, s_bp);
        }
    } else {
        constexpr int PER = VEC == 8 ? 4 : 1;
        typedef float piece __attribute__((ext_vector_type(PER)));
        __syncthreads();                         // the parameters have been read
        const Shared mine{joined + team * (SUMS * Shared::SIZE)};
        const auto leave = [&](int kind, const float (&f)[CH][VEC]) { Shared{mine.at0 + kind * Shared::SIZE}.put(f, lane); };
        leave(0, s_g);
        leave(1, s_wq);
        leave(2, s_bq);
        if constexpr (POST) {
            leave(3, s_wp);
            leave(4, s_bp);
        }
        __syncthreads();
        for (int q = threadIdx.x; q < SUMS * Shared::SIZE / PER; q += TEAMS * LANES) {
            const int kind = q / (Shared::SIZE / PER), place = q % (Shared::SIZE / PER), ch = Shared::channel(place);
            if (ch >= a.d || !dst[kind]) continue;
            piece sum = *(const piece *)(joined + q * PER);
#pragma unroll
            for (int t = 1; t < TEAMS; ++t) sum += *(const piece *)(joined + t * (SUMS * Shared::SIZE) + q * PER);
            *(piece *)(parts + kind * span + ch) = sum;
        }
    }
}

// Adds what the workgroups and runs left, in a fixed order.  Blocks 0 .. 5 *
// col_blocks - 1 take one kind of sum and 16 channels each, 64 groups of 16 lanes
// going through the workgroups in turn.  The others join the gate groups that several
// runs share: few groups, of many runs each, 64 channels a workgroup, 16 waves going through
// the runs; many groups (MANY: under 16 runs each), 256 channels a wave.  Such a group
// holds the first row of a run, so where there are more groups than runs those of the
// runs' first rows are enough.  256 workgroups' sums of 1024 channels: 5.2 MB, 4.0 us.  The
// whole backward pass of 18464 x 1024 bf16 with 1154 groups takes 54 us (a workgroup for each
// group and 64 channels: 105), with a group a token 85 (858).
template <int WIDE>
__device__ __forceinline__ void add_turns(float *part, float s, float *dst, bool in) {
    constexpr int TURNS = 1024 / WIDE;
    const int turn = threadIdx.x / WIDE, lane = threadIdx.x % WIDE;
    part[turn * (WIDE + 1) + lane] = s;
    __syncthreads();
    if (turn < TURNS / 16) {
        float sum = 0.f;
#pragma unroll
        for (int w = 0; w < 16; ++w) sum += part[(turn * 16 + w) * (WIDE + 1) + lane];
        part[turn * 16 * (WIDE + 1) + lane] = sum;
    }
    __syncthreads();
    if (turn == 0 && in) {
        float sum = 0.f;
#pragma unroll
        for (int w = 0; w < TURNS / 16; ++w) sum += part[w * 16 * (WIDE + 1) + lane];
        *dst = sum;
    }
}

template <bool MANY>
__global__ __launch_bounds__(1024) void k_norm_sums(NormGradArgs a, int workgroups, int col_blocks) {
    __shared__ float part[64 * 17];
    float s = 0.f;
    if ((int)blockIdx.x < 5 * col_blocks) {
        const int kind = blockIdx.x / col_blocks, turn = threadIdx.x >> 4;
        const int ch = (blockIdx.x % col_blocks) * 16 + (threadIdx.x & 15);
        float *dst = kind == 0 ? (a.groups <= 1 ? a.dgate : nullptr) : kind == 1 ? a.dpre_weight : kind == 2 ? a.dpre_bias
                     : kind == 3 ? a.dpost_weight : a.dpost_bias;
        if (!dst) return;
        if (ch < a.d) {
            const float *src = a.parts + (int64_t)kind * workgroups * a.d + ch;
#pragma unroll 8
            for (int w = turn; w < workgroups; w += 64) s += src[(int64_t)w * a.d];
        }
        add_turns<16>(part, s, dst + ch, ch < a.d);
    } else {
        const int b = blockIdx.x - 5 * col_blocks;
        const int wide = MANY ? (a.d + 255) / 256 : (a.d + 63) / 64;
        const int item = MANY ? b * 16 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) : b;
        const bool by_run = MANY && a.groups >= a.runs;
        const int place = item / wide, group = by_run ? first_row(place + 1, a.m, a.runs) / a.per_group : place;
        if (MANY && place >= (by_run ? a.runs - 1 : a.groups)) return;
        const int t0 = run_of(group * a.per_group, a.m, a.runs), t1 = run_of((group + 1) * a.per_group - 1, a.m, a.runs);
        if (t0 == t1) return;              // within one run: finished there
        if (by_run && t0 != place) return; // begins in another run, whose end has it (or a later one's)
        const auto left = [&](int t) {
            return a.gate_parts + ((int64_t)2 * t + (group == first_row(t, a.m, a.runs) / a.per_group ? 0 : 1)) * a.d;
        };
        float *dst = a.dgate + (int64_t)group * a.d;
        if constexpr (MANY) {
            const int ch0 = item % wide * 256 + (threadIdx.x & 63);
            float sum[4] = {};
            for (int t = t0; t <= t1; ++t) {
                const float *src = left(t);
#pragma unroll
                for (int q = 0; q < 4; ++q)
                    if (ch0 + q * 64 < a.d) sum[q] += src[ch0 + q * 64];
            }
#pragma unroll
            for (int q = 0; q < 4; ++q)
                if (ch0 + q * 64 < a.d) dst[ch0 + q * 64] = sum[q];
        } else {
            const int ch = item % wide * 64 + (threadIdx.x & 63);
            if (ch < a.d)
                for (int t = t0 + (threadIdx.x >> 6); t <= t1; t += 16) s += left(t)[ch];
            add_turns<64>(part, s, dst + ch, ch < a.d);
        }
    }
}

// --------------------------------------------------------------- row codes
// One team for each row; a row past 16 values a lane is read a second time
// (from L2) for its codes.  Bound by memory: 18464 x 1024 fp16 12.2 to 12.9 us, 4.5 TB/s.
template <class T, int VEC, int CH, int WPR>
__global__ __launch_bounds__(team_threads(WPR)) void k_quantize_rows(QuantArgs a) {
    constexpr int TEAMS = team_threads(WPR) / 64 / WPR;
    __shared__ float box[TEAMS][2][2][WPR];
    const int team = __builtin_amdgcn_readfirstlane(threadIdx.x / (64 * WPR)), lane = threadIdx.x % (64 * WPR);
    RowReduce<WPR> red{box[team], lane >> 6};
    const int step = 64 * WPR * VEC, span = step * CH;
    for (int64_t row0 = (int64_t)blockIdx.x * TEAMS; row0 < a.m; row0 += (int64_t)gridDim.x * TEAMS) {
        const int64_t row = row0 + team;
        const bool live = row < a.m;
        const __amdgpu_buffer_rsrc_t src = row_of(a.x, (live ? row : 0) * a.ldx * (int)sizeof(T), a.k * (int)sizeof(T));
        Part<T, VEC, CH> p;
        float top = 0.f;
        int base = 0;
        for (;; base += span) {
            load_part(p, src, base + lane * VEC, step);
            float f[CH][VEC];
            p.get(f);
#pragma unroll
            for (int c = 0; c < CH; ++c)
#pragma unroll
                for (int e = 0; e < VEC; ++e) top = larger(top, magnitude(f[c][e]));
            if (base + span >= a.ldq) break;
        }
        const RowScale rs = row_scale(red.largest(top));
        if (live && lane == 0) a.scale[row] = rs.scale;
        for (;; base -= span) {      // the last part is still in registers
            float f[CH][VEC];
            p.get(f);
#pragma unroll
            for (int c = 0; c < CH; ++c) {
                const int ch = base + lane * VEC + c * step;
                if (!live || ch >= a.ldq) continue;
                int8_t *dst = a.q + row * a.ldq + ch;
                int q[VEC];
#pragma unroll
                for (int e = 0; e < VEC; ++e) q[e] = row_code(f[c][e], rs.inv);
                if constexpr (VEC == 8)
                    *(v2u *)dst = v2u{pack4(q[0], q[1], q[2], q[3]), pack4(q[4], q[5], q[6], q[7])};
                else
                    *dst = (int8_t)q[0];
            }
            if (base == 0) break;
            load_part(p, src, base - span + lane * VEC, step);
        }
    }
}

// One 16-byte piece of a padded row a thread, from any address.
__global__ __launch_bounds__(256) void k_pad_codes(PadArgs a) {
    typedef unsigned int v4u_bytes __attribute__((ext_vector_type(4), aligned(1)));
    const int64_t per = a.ldo / 16, pieces = a.m * per;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < pieces; i += (int64_t)gridDim.x * 256) {
        const int64_t row = i / per;
        const int c = (int)(i - row * per) * 16;
        const int8_t *src = a.q + row * a.ldq + c;
        v4u v = {0, 0, 0, 0};
        if (c + 16 <= a.k) {
            v = *(const v4u_bytes *)src;
        } else {
            for (int e = 0; e < a.k - c; ++e) v[e / 4] |= (unsigned)(uint8_t)src[e] << (e % 4 * 8);
        }
        *(v4u *)(a.out + i * 16) = v;
    }
}

// --------------------------------------------------------------- launches
// Waves of a team by the row's length, and workgroups that the device holds at once.
constexpr int kResident = 8;

template <class T, int VEC, int CH, int WPR>
int norm_one(const NormArgs &a, void *stream) {
    constexpr int teams = team_threads(WPR) / 64 / WPR;
    const int64_t want = ((int64_t)a.m + teams - 1) / teams, most = (int64_t)device_cu_count() * kResident;
    hipLaunchKernelGGL((k_norm_residual<T, VEC, CH, WPR>), dim3((unsigned)(want < most ? want : most)),
                       dim3(team_threads(WPR)), 0, (hipStream_t)stream, a);
    return (int)hipGetLastError();
}
template <class T, int VEC>
int norm_by_width(const NormArgs &a, void *stream) {
    constexpr int full = 16 / VEC;
    const int w = a.zq ? (int)a.ldq : a.d;
    if (w <= 512) return norm_one<T, VEC, full / 2, 1>(a, stream);
    if (w <= 1024) return norm_one<T, VEC, full, 1>(a, stream);
    if (w <= 2048) return norm_one<T, VEC, full, 2>(a, stream);
    if (w <= 4096) return norm_one<T, VEC, full, 4>(a, stream);
    if (w <= 8192) return norm_one<T, VEC, full, 8>(a, stream);
    return norm_one<T, VEC, full, 16>(a, stream);
}

template <class T, int VEC, int CH, int WPR, bool POST>
int grad_one(const NormGradArgs &a, int workgroups, void *stream) {
    hipLaunchKernelGGL((k_norm_residual_backward<T, VEC, CH, WPR, POST>), dim3(workgroups),
                       dim3(64 * WPR * grad_teams(WPR, VEC, CH, POST)), 0, (hipStream_t)stream, a);
    return (int)hipGetLastError();
}
template <class T, int VEC, bool POST>
int grad_by_width(const NormGradArgs &a, int workgroups, void *stream) {
    constexpr int half = 8 / VEC;
    if (a.d <= 512) return grad_one<T, VEC, half, 1, POST>(a, workgroups, stream);
    if (a.d <= 1024) return grad_one<T, VEC, half, 2, POST>(a, workgroups, stream);
    if (a.d <= 2048) return grad_one<T, VEC, half, 4, POST>(a, workgroups, stream);
    if (a.d <= 4096) return grad_one<T, VEC, half, 8, POST>(a, workgroups, stream);
    // 16 waves leave a wave 128 registers: with both norms' sums 8 waves of twice the
    // channels are faster (2048 x 8192 bf16: 73 us against 139)
    constexpr bool wide = VEC == 8 && POST;
    if (a.d <= 8192) return grad_one<T, VEC, wide ? 2 * half : half, wide ? 8 : 16, POST>(a, workgroups, stream);
    return grad_one<T, VEC, 2 * half, 16, POST>(a, workgroups, stream);
}
template <class T>
int grad_of(bool vec, const NormGradArgs &a, int workgroups, void *stream) {
    const bool post = a.post.kind != NM_NORM_NONE && a.y;
    if (vec) return post ? grad_by_width<T, 8, true>(a, workgroups, stream) : grad_by_width<T, 8, false>(a, workgroups, stream);
    return post ? grad_by_width<T, 1, true>(a, workgroups, stream) : grad_by_width<T, 1, false>(a, workgroups, stream);
}

template <class T, int VEC, int CH, int WPR>
int quant_one(const QuantArgs &a, void *stream) {
    constexpr int teams = team_threads(WPR) / 64 / WPR;
    const int64_t want = (a.m + teams - 1) / teams, most = (int64_t)device_cu_count() * 2 * kResident;
    hipLaunchKernelGGL((k_quantize_rows<T, VEC, CH, WPR>), dim3((unsigned)(want < most ? want : most)),
                       dim3(team_threads(WPR)), 0, (hipStream_t)stream, a);
    return (int)hipGetLastError();
}
template <class T, int VEC>
int quant_by_width(const QuantArgs &a, void *stream) {
    constexpr int full = 16 / VEC;
    if (a.ldq <= 512) return quant_one<T, VEC, full / 2, 1>(a, stream);
    if (a.ldq <= 1024) return quant_one<T, VEC, full, 1>(a, stream);
    if (a.ldq <= 2048) return quant_one<T, VEC, full, 2>(a, stream);
    return quant_one<T, VEC, full, 4>(a, stream);
}

}  // namespace

// Workgroups of the backward kernel for m rows, one a compute unit, and the rows of a
// run: as many as another's or one more.
NormGradShape norm_grad_shape(int m, int d, bool vec, bool post) {
    const int v = vec ? 8 : 1, half = 8 / v;
    const int wpr = d <= 512 ? 1 : d <= 1024 ? 2 : d <= 2048 ? 4 : d <= 4096 || (d <= 8192 && vec && post) ? 8 : 16;
    const int ch = d > 8192 || (d > 4096 && vec && post) ? 2 * half : half;
    const int teams = grad_teams(wpr, v, ch, post), most = device_cu_count(), want = (m + teams - 1) / teams;
    NormGradShape s;
    s.workgroups = want < most ? want : most;
    s.runs = s.workgroups * teams < m ? s.workgroups * teams : m;
    s.turns = (m + s.runs - 1) / s.runs;
    return s;
}

int launch_norm_residual(int type, bool vec, const NormArgs &a, void *stream) {
    switch (type) {
        case NM_TYPE_F16: return vec ? norm_by_width<half_t, 8>(a, stream) : norm_by_width<half_t, 1>(a, stream);
        case NM_TYPE_BF16: return vec ? norm_by_width<bf16_t, 8>(a, stream) : norm_by_width<bf16_t, 1>(a, stream);
        case NM_TYPE_F32: return vec ? norm_by_width<float, 8>(a, stream) : norm_by_width<float, 1>(a, stream);
    }
    return (int)hipErrorInvalidValue;
}

int launch_norm_residual_backward(int type, bool vec, const NormGradArgs &a, int workgroups, void *stream) {
    int err = (int)hipErrorInvalidValue;
    switch (type) {
        case NM_TYPE_F16: err = grad_of<half_t>(vec, a, workgroups, stream); break;
        case NM_TYPE_BF16: err = grad_of<bf16_t>(vec, a, workgroups, stream); break;
        case NM_TYPE_F32: err = grad_of<float>(vec, a, workgroups, stream); break;
    }
    if (err != 0) return err;
    const int col_blocks = (a.d + 15) / 16;
    const bool shared = a.groups > 1 && a.dgate, many = shared && a.runs < 16 * (int64_t)a.groups;
    const int places = a.groups < a.runs ? a.groups : a.runs - 1;     // where shared groups are looked for
    if (many)
        hipLaunchKernelGGL(k_norm_sums<true>, dim3(5 * col_blocks + (places * ((a.d + 255) / 256) + 15) / 16), dim3(1024),
                           0, (hipStream_t)stream, a, workgroups, col_blocks);
    else
        hipLaunchKernelGGL(k_norm_sums<false>, dim3(5 * col_blocks + (shared ? places * ((a.d + 63) / 64) : 0)),
                           dim3(1024), 0, (hipStream_t)stream, a, workgroups, col_blocks);
    return (int)hipGetLastError();
}

int launch_pad_codes(const PadArgs &a, void *stream) {
    const int64_t want = (a.m * (a.ldo / 16) + 255) / 256, most = (int64_t)device_cu_count() * kResident;
    hipLaunchKernelGGL(k_pad_codes, dim3((unsigned)(want < most ? want : most)), dim3(256), 0, (hipStream_t)stream, a);
    return (int)hipGetLastError();
}

int launch_quantize_rows(int type, bool vec, const QuantArgs &a, void *stream) {
    switch (type) {
        case NM_TYPE_F16: return vec ? quant_by_width<half_t, 8>(a, stream) : quant_by_width<half_t, 1>(a, stream);
        case NM_TYPE_BF16: return vec ? quant_by_width<bf16_t, 8>(a, stream) : quant_by_width<bf16_t, 1>(a, stream);
        case NM_TYPE_F32: return vec ? quant_by_width<float, 8>(a, stream) : quant_by_width<float, 1>(a, stream);
    }
    return (int)hipErrorInvalidValue;
}

}  // namespace nmspmm
