// Device code shared by the kernels of differential attention: tiles of rows in
// LDS, operands of the 32 x 32 x 16 matrix instruction from them, the extent of
// a sequence and what its rows see.
//
// Operand maps (a lane is l, half h = l / 32, column or row r = l % 32):
//   A, B: 8 values of row (A) or column (B) r at k = 8 h .. 8 h + 7
//   C:    column r, value e of 16 at row 8 (e / 4) + 4 h + e % 4
// So the rows of C that a lane holds in values 8 c .. 8 c + 7 are the quads 16 c + 4 h
// and 16 c + 8 + 4 h: rounded to 16 bits they are a B operand of 16 rows of k as they
// lie, if the A operand takes its k in the same order.  turned() reads A that way
// from rows in LDS, so no value of the maps crosses lanes.
#pragma once

#include <hip/hip_runtime.h>

#include <type_traits>

#include "nmspmm_attn_internal.h"
#include "nmspmm_values.h"

namespace nmspmm {
namespace {

typedef float v16f __attribute__((ext_vector_type(16)));
typedef float v4f __attribute__((ext_vector_type(4)));
typedef int v4i __attribute__((ext_vector_type(4)));
typedef short v4s __attribute__((ext_vector_type(4)));
typedef short v8s __attribute__((ext_vector_type(8)));

template <class T>
struct Mfma;
template <>
struct Mfma<half_t> {
    typedef half_t v8 __attribute__((ext_vector_type(8)));
    static __device__ __forceinline__ v16f mul(v8s a, v8s b, v16f c) {
        return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(v8, a), __builtin_bit_cast(v8, b), c, 0, 0, 0);
    }
};
template <>
struct Mfma<bf16_t> {
    typedef bf16_t v8 __attribute__((ext_vector_type(8)));
    static __device__ __forceinline__ v16f mul(v8s a, v8s b, v16f c) {
        return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(v8, a), __builtin_bit_cast(v8, b), c, 0, 0, 0);
    }
};

// Eight values of C (8 c .. 8 c + 7), rounded once: a B operand.
template <class T>
__device__ __forceinline__ v8s pack(const float (&f)[8]) {
    typedef T v8 __attribute__((ext_vector_type(8)));
    v8 r;
#pragma unroll
    for (int e = 0; e < 8; ++e) r[e] = (T)f[e];
    return __builtin_bit_cast(v8s, r);
}

// Sum and larger of a lane's value and that of the lane 32 away, in both.
__device__ __forceinline__ float half_sum(float x) {
    const uint32_t u = __builtin_bit_cast(uint32_t, x);
    const auto r = __builtin_amdgcn_permlane32_swap(u, u, false, false);
    return __builtin_bit_cast(float, (uint32_t)r[0]) + __builtin_bit_cast(float, (uint32_t)r[1]);
}
__device__ __forceinline__ float half_max(float x) {
    const uint32_t u = __builtin_bit_cast(uint32_t, x);
    const auto r = __builtin_amdgcn_permlane32_swap(u, u, false, false);
    return fmaxf(__builtin_bit_cast(float, (uint32_t)r[0]), __builtin_bit_cast(float, (uint32_t)r[1]));
}

// ---------------------------------------------------------------- tiles in LDS
// LDS is addressed by bytes from its start.
template <class V>
__device__ __forceinline__ V lds_load(uint32_t at) {
    return *(const __attribute__((address_space(3))) V *)(uintptr_t)at;
}
__device__ __forceinline__ uint32_t lds_start(char *lds) {
    return (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char *)lds;
}

// 16 or 4 bytes a lane straight to LDS, lane l's at lds + 16 l or 4 l (lds wave-uniform), from a uniform base
// and a lane's offset, or from a lane's address.  M0 holds the LDS address; the wait states cover its write and a
// vector instruction's write of the base's registers.
__device__ __forceinline__ uint32_t uniform(uint32_t x) { return (uint32_t)__builtin_amdgcn_readfirstlane((int)x); }
__device__ __forceinline__ const void *uniform(const void *p) {
    const uint64_t at = (uint64_t)p;
    return (const void *)((uint64_t)uniform((uint32_t)(at >> 32)) << 32 | uniform((uint32_t)at));
}
__device__ __forceinline__ void dma16(const void *base, uint32_t offset, uint32_t lds) {
    asm volatile("s_mov_b32 m0, %2\n\ts_nop 4\n\tglobal_load_lds_dwordx4 %0, %1" ::"v"(offset), "s"(base), "s"(uniform(lds))
                 : "memory", "m0");
}
__device__ __forceinline__ void dma16(const void *at, uint32_t lds) {
    asm volatile("s_mov_b32 m0, %1\n\ts_nop 4\n\tglobal_load_lds_dwordx4 %0, off" ::"v"(at), "s"(uniform(lds)) : "memory", "m0");
}
__device__ __forceinline__ void dma4(const void *at, uint32_t lds) {
    asm volatile("s_mov_b32 m0, %1\n\ts_nop 4\n\tglobal_load_lds_dword %0, off" ::"v"(at), "s"(uniform(lds)) : "memory", "m0");
}
// What lanes load whose piece is behind a tensor's rows or columns.
__device__ const int zeros[4] __attribute__((aligned(16))) = {0, 0, 0, 0};
// All of this wave's loads have arrived, then the workgroup's barrier.
__device__ __forceinline__ void arrive() {
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_waitcnt(0);
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
}

// This wave's loads have arrived, in LDS that no other wave reads.
__device__ __forceinline__ void arrive_alone() {
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_waitcnt(0);
    asm volatile("" ::: "memory");
}

// ROWS rows of CPR 16-byte pieces in LDS.  One load of a wave fills 1024 bytes, a group of
// 64 / CPR rows.  Which rows make a group, and a gap of 16 bytes for each step of a group's
// number, put the rows of an operand (16 lanes at one piece) and the 4 rows of a turned one
// (32 lanes at 64 bytes of each) in distinct banks.  A row's place is a sum over the bits of its
// number, so an operand is read at one address of its lane and constants.
template <class T, int CPR, int ROWS, int WAVES>
struct Tile {
    static constexpr int GROUPS = ROWS * CPR / 64;
    static_assert(ROWS == 32 || ROWS == 64 || ROWS == 128, "rows");
    // bits of a row's number in the place within its group, then in the group's number, from the lowest
    static constexpr int order(int n) {
        constexpr int few[4][6] = {{0, 1, 4, 3, 2, 5}, {1, 4, 3, 2, 0, 5}, {4, 3, 2, 0, 1, 5}, {4, 2, 3, 0, 1, 5}};
        constexpr int many[4][6] = {{0, 1, 4, 5, 2, 3}, {1, 4, 5, 2, 3, 0}, {4, 5, 2, 3, 0, 1}, {4, 2, 3, 0, 1, 5}};
        constexpr int kind = CPR == 4 ? 0 : CPR == 8 ? 1 : CPR == 16 ? 2 : 3;
        return n == 6 ? 6 : ROWS == 32 ? few[kind][n] : many[kind][n];
    }
    static constexpr int PLACE_BITS = CPR == 4 ? 4 : CPR == 8 ? 3 : CPR == 16 ? 2 : 1;
    // 16-byte steps of a group's gap
    static constexpr int gap(int group) {
        if (ROWS == 32 && CPR == 8) return (group & 1) + (group >> 1 & 1) * 4;
        if (ROWS == 32 && CPR == 16) return (group & 1) + (group >> 1 & 1) * 4 + (group >> 2 & 1) * 8;
        return group;
    }
    static constexpr int BYTES = GROUPS * 1024 + (gap(GROUPS - 1) * 16 + 127) / 128 * 128;
    static constexpr __host__ __device__ int group_at(int group) { return group * 1024 + gap(group) * 16; }
    // where a row lies, and the rows of a group and place
    static constexpr __host__ __device__ int place_of(int row) {
        int place = 0, group = 0;
        for (int n = 0; n < 7; ++n) {
            const int bit = row >> order(n) & 1;
            if (n < PLACE_BITS)
                place |= bit << n;
            else
                group |= bit << (n - PLACE_BITS);
        }
        return group_at(group) + place * CPR * 16;
    }
    static constexpr __host__ __device__ int row_of_place(int place) {
        int row = 0;
        for (int n = 0; n < PLACE_BITS; ++n) row |= (place >> n & 1) << order(n);
        return row;
    }
    static constexpr __host__ __device__ int row_of_group(int group) {
        int row = 0;
        for (int n = PLACE_BITS; n < 7; ++n) row |= (group >> (n - PLACE_BITS) & 1) << order(n);
        return row;
    }

    // The A or B operand of the rows row .. row + 31 (row: a multiple of 32), k = 16 c .. 16 c + 15, at
    // the address of this lane's part of it.
    static __device__ __forceinline__ uint32_t rows_lane(int lane) { return place_of(lane & 31) + (lane >> 5) * 16; }
    static __device__ __forceinline__ v8s rows(uint32_t at, int row, int c) {
        return lds_load<v8s>(at + (place_of(row) + c * 32));
    }
    // The A operand of 32 columns from 32 x with k over the rows row .. row + 15 (row: a
    // multiple of 16) in the order that values of C have (above).  A read gives 16 lanes 4 rows x 16
    // columns: lane i gives the address of 4 columns of row i / 4 and gets the 4 rows of column i.
    static __device__ __forceinline__ uint32_t turned_lane(int lane) {
        return place_of((lane & 15) >> 2 | (lane >> 5) << 2) + (lane >> 4 & 1) * 32 + (lane & 3) * 8;
    }
    static __device__ __forceinline__ v8s turned(uint32_t at, int row, int x) {
        const v4s a = read4(at + (place_of(row) + x * 64)), b = read4(at + (place_of(row + 8) + x * 64));
        return __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7);
    }
    static __device__ __forceinline__ v4s read4(uint32_t at) {
        return __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) v4s *)(uintptr_t)at);
    }
};

// Values c .. c + 7 of a row of `width`, c < width, zero from there on, at any alignment of its type (the hardware's
// loads take it).  A row's last values are the end of its last 8, which moved() brings to their places: `over` of them
// lie before the piece.
__device__ __forceinline__ int piece_over(int c, int width) { return width >= 8 && c + 8 > width ? c + 8 - width : 0; }
template <class T>
__device__ __forceinline__ v8s row_piece(const T *row, int c, int width, int over) {
    typedef short v8any __attribute__((ext_vector_type(8), aligned(2)));
    const short *p = (const short *)row;
    if (width >= 8) return *(const v8any *)(p + c - over);
    v8s v = {};
#pragma unroll
    for (int e = 0; e < 7; ++e)
        if (c + e < width) v[e] = p[c + e];
    return v;
}
__device__ __forceinline__ v8s moved(v8s v, int over) {        // 0 < over < 8
    typedef uint64_t v2l __attribute__((ext_vector_type(2)));
    const v2l x = __builtin_bit_cast(v2l, v);
    const int bits = 16 * over;
    const v2l y = bits >= 64 ? v2l{x[1] >> (bits - 64), 0} : v2l{x[0] >> bits | x[1] << (64 - bits), x[1] >> bits};
    return __builtin_bit_cast(v8s, y);
}

// Loads of tile after tile of rows, of one tensor or of two `second` values apart (their tiles one behind the
// other): rows behind the last and columns from `width` on are zero, whatever memory holds there.  PIECES: in whole
// pieces at 16-byte boundaries the loads go straight to LDS and arrive later (LOADS of them by every
// wave); otherwise through registers, at once, by kernels of their own (beside the others' they cost spilled
// registers).  What a load needs but its tile's base is made once.
template <class T, int CPR, int ROWS, int WAVES, int TENSORS, bool PIECES>
struct Feed {
    using Place = Tile<T, CPR, ROWS, WAVES>;
    static constexpr int GROUPS = Place::GROUPS, LOADS = TENSORS * GROUPS / WAVES;
    static constexpr bool SPREAD = GROUPS < WAVES;          // waves share out the tensors too
    static constexpr int EACH = SPREAD ? 1 : GROUPS / WAVES; // loads of one tensor
    static_assert(TENSORS * GROUPS % WAVES == 0 && (SPREAD || GROUPS % WAVES == 0), "as many loads by every wave");
    const T *p;
    int64_t stride, second;
    int left, width, first;             // rows left; this wave's first group
    uint32_t offset[EACH];              // of a lane, in bytes
    __device__ __forceinline__ Feed(const T *from, int64_t row_stride, int64_t tensor_stride, int rows, int columns, int wave,
                                    int lane)
        : p(from), stride(row_stride), second(tensor_stride), left(rows), width(columns) {
        first = SPREAD ? wave % GROUPS : wave;
        if (SPREAD) p += wave / GROUPS * second;
        const int c = lane % CPR;
#pragma unroll
        for (int i = 0; i < EACH; ++i)
            offset[i] = (uint32_t)(Place::row_of_place(lane / CPR) + Place::row_of_group(i * WAVES + first)) *
                            (uint32_t)stride * 2 + c * 16;
    }
    __device__ __forceinline__ void load(uint32_t lds, int wave, int lane) {
        if (SPREAD) lds += wave / GROUPS * Place::BYTES;
        if constexpr (PIECES) {
            if (left >= ROWS && width == CPR * 8) {
#pragma unroll
                for (int t = 0; t < (SPREAD ? 1 : TENSORS); ++t) {
                    const void *from = uniform(p + t * second);
#pragma unroll
                    for (int i = 0; i < EACH; ++i)
                        dma16(from, offset[i], lds + t * Place::BYTES + Place::group_at(i * WAVES + first));
                }
            } else {
                const bool column = lane % CPR * 8 < width;
#pragma unroll
                for (int n = 0; n < LOADS; ++n) {
                    const int t = n / EACH, group = n % EACH * WAVES + first;
                    const int row = Place::row_of_place(lane / CPR) + Place::row_of_group(group);
                    const char *at = (const char *)(p + t * second) + offset[n % EACH];
                    dma16(column && row < left ? at : (const char *)zeros, lds + t * Place::BYTES + Place::group_at(group));
                }
            }
        } else {
            constexpr int BATCH = LOADS < 8 ? LOADS : 8;        // loads under way together
            const int c = lane % CPR * 8, over = piece_over(c, width);
#pragma unroll 1
            for (int n = 0; n < LOADS; n += BATCH) {
                v8s v[BATCH];
#pragma unroll
                for (int i = 0; i < BATCH; ++i) {
                    const int t = (n + i) / EACH, group = (n + i) % EACH * WAVES + first;
                    const int row = Place::row_of_group(group) + Place::row_of_place(lane / CPR);
                    v[i] = v8s{};
                    if (row < left && c < width) v[i] = row_piece(p + t * second + row * stride, c, width, over);
                }
                if (over > 0)
#pragma unroll
                    for (int i = 0; i < BATCH; ++i) v[i] = moved(v[i], over);
#pragma unroll
                for (int i = 0; i < BATCH; ++i) {
                    const int t = (n + i) / EACH, group = (n + i) % EACH * WAVES + first;
                    *(__attribute__((address_space(3))) v8s *)(uintptr_t)(lds + t * Place::BYTES + Place::group_at(group) +
                                                                         lane * 16) = v[i];
                }
            }
        }
        p += ROWS * stride;
        left -= ROWS;
    }
};

// The B operand of a row in memory, k = 16 c .. 16 c + 15, zero from `width` on; PIECES as above.
template <bool PIECES, class T>
__device__ __forceinline__ v8s row_operand(const T *p, bool valid, int c, int width, int lane) {
    const int at = 16 * c + 8 * (lane >> 5);
    if (!valid || at >= width) return v8s{};
    if constexpr (PIECES) return *(const v8s *)(p + at);
    const int over = piece_over(at, width);
    const v8s v = row_piece(p, at, width, over);
    return over > 0 ? moved(v, over) : v;
}

// 4 values of a row at column c of `width`, at any alignment of their type.
template <class T, class X>
__device__ __forceinline__ void store4(T *p, int c, int width, X a, X b, X d, X e) {
    typedef T v4 __attribute__((ext_vector_type(4), aligned(sizeof(T))));
    if (c + 4 <= width) {
        *(v4 *)(p + c) = v4{(T)a, (T)b, (T)d, (T)e};
        return;
    }
    if (c < width) p[c] = (T)a;
    if (c + 1 < width) p[c + 1] = (T)b;
    if (c + 2 < width) p[c + 2] = (T)d;
}

// Codes in 16 bits of values of which `top` is the largest magnitude: what the backward pass
// keeps of both maps' products, whose sums with do are differences' small parts.
struct KeptScale {
    float scale, inv;
};
__device__ __forceinline__ KeptScale kept_scale(float top) {
    if (!(top < __builtin_inff())) return {__builtin_nanf(""), 0.f};
    if (top < 0x1p-100f) return {0.f, 0.f};
    return {top * (1.f / 32767.f), 32767.f / top};
}
__device__ __forceinline__ short kept_code(float x, float inv) {
    int r;
    asm("v_cvt_i32_f32 %0, %1" : "=v"(r) : "v"(__builtin_rintf(x * inv)));
    return (short)r;
}

// Powers of two that take small values up before a rounding to binary16, whose exponents end at 2^-14 and whose
// steps at 2^-24: gradients of scores over thousands of keys lie below both.  bfloat16 has binary32's exponents.
template <class T>
constexpr bool kFewExponents = std::is_same<T, half_t>::value;
// The forward pass's maps and their sums are 2^this of themselves.
template <class T>
constexpr float kMapsUp = kFewExponents<T> ? 7.f : 0.f;
__device__ __forceinline__ float power(int e) { return __builtin_bit_cast(float, (uint32_t)(127 + e) << 23); }
// x >= 0 is below 2^exponent(x), the exponent held within lo .. hi (infinities and NaN: hi)
__device__ __forceinline__ int exponent(float x, int lo, int hi) {
    const int e = (int)(__builtin_bit_cast(uint32_t, x) >> 23) - 126;
    return e < lo ? lo : e > hi ? hi : e;
}
__device__ __forceinline__ int half_up(int e) { return (e + 1) >> 1; }        // of a square's exponent: x^2 < 2^e, x < 2^this
__device__ __forceinline__ float inverse(float power) {
    return __builtin_bit_cast(float, (254u << 23) - __builtin_bit_cast(uint32_t, power));
}

// ---------------------------------------------------------------- sequences

// A sequence: its lengths, its tensors' first rows and the number of its first row.
// Lengths and offsets come from device memory: they are held within the tensors.
struct Sequence {
    int nq, nk;
    int64_t q0, k0;   // rows before it in packed tensors (else the batch's stride tells)
    int64_t row0;
    int batch;        // 0 where packed
};
__device__ __forceinline__ int64_t within(int64_t v, int64_t lo, int64_t hi) { return v < lo ? lo : v > hi ? hi : v; }
__device__ __forceinline__ Sequence sequence(const AttnArgs &a, int b) {
    Sequence s;
    s.q0 = s.k0 = 0;
    s.nq = a.tq;
    s.nk = a.tk;
    s.row0 = (int64_t)b * a.tq;
    s.batch = b;
    if (a.q_offsets) {
        s.q0 = within(a.q_offsets[b], 0, a.total_q);
        s.nq = (int)within(within(a.q_offsets[b + 1], s.q0, a.total_q) - s.q0, 0, a.tq);
        s.k0 = within(a.k_offsets[b], 0, a.total_k);
        s.nk = (int)within(within(a.k_offsets[b + 1], s.k0, a.total_k) - s.k0, 0, a.tk);
        s.row0 = s.q0;
        s.batch = 0;
    } else {
        if (a.q_lens) s.nq = (int)within(a.q_lens[b], 0, a.tq);
        if (a.k_lens) s.nk = (int)within(a.k_lens[b], 0, a.tk);
    }
    return s;
}
template <class T>
__device__ __forceinline__ T *head_of(const Heads &t, int batch, int64_t row, int head) {
    return (T *)t.p + batch * t.batch + row * t.token + head * t.head;
}

// First and last key that row t sees (last < first: none).
__device__ __forceinline__ int first_seen(const AttnArgs &a, const Sequence &s, int t) {
    const int at = t + s.nk - s.nq - a.left;
    return at > 0 ? at : 0;
}
__device__ __forceinline__ int last_seen(const AttnArgs &a, const Sequence &s, int t) {
    const int at = t + s.nk - s.nq + a.right;
    return at < s.nk - 1 ? at : s.nk - 1;
}

// lam of a head, by the whole wave: given, or exp(q1 . k1) - exp(q2 . k2) + init.
struct Weight {
    float lam, e1, e2;
};
__device__ __forceinline__ Weight weight_of(const nm_diff_weight &w, int head, int lane) {
    Weight r = {0.f, 0.f, 0.f};
    if (w.value) {
        r.lam = w.value[head];
        return r;
    }
    const int64_t at = w.per_head ? (int64_t)head * w.n : 0;
    float a = 0.f, b = 0.f;
    for (int i = lane; i < w.n; i += 64) {
        a += w.q1[at + i] * w.k1[at + i];
        b += w.q2[at + i] * w.k2[at + i];
    }
    r.e1 = expf(wave_sum(a));
    r.e2 = expf(wave_sum(b));
    r.lam = r.e1 - r.e2 + w.init;
    return r;
}

// Workgroups are dispatched round-robin over the 8 XCDs; those of one head (which share its
// keys) run on one of them, whose L2 then holds the keys.  Under a causal mask work falls along
// a head's tiles: the second 32 of an XCD (which has 32 compute units) go backwards, so that
// the two workgroups that a compute unit starts with are a long and a short one (2 x 4096 causal rows of
// 8 heads, forward: 151 us, in order 172).  The kernel of dk and dv has one workgroup a compute unit and loses by
// it: there the backward pass takes 388 us and in order 349.
__device__ __forceinline__ int near_block(int bid, int count) {
    const int xcd = bid & 7, per = count >> 3, left = count & 7;
    const int mine = xcd < left ? per + 1 : per, before = xcd < left ? xcd * (per + 1) : left * (per + 1) + (xcd - left) * per;
    int local = bid >> 3;
    if (local >> 5 == 1) {
        const int from = 32, to = mine < 64 ? mine : 64;
        local = from + to - 1 - local;
    }
    return before + local;
}

// The rows of a workgroup: `TILE` of the rows (token t, head g of the group) number t * group + g that
// share a key head, 32 a block; a lane's row is the block's number lane % 32.
struct RowTile {
    Sequence s;
    int b, hk, tile, start, rows;
    bool valid;           // lanes behind the last row repeat it and store nothing
    int t, g, head;
    int first, last;      // keys that the lane's row sees
    // what the block's rows see, one of them or all: rows rise with t, and so do both ends
    int block_low, block_high, block_full, block_end;
    int low, high;        // what the workgroup's rows see
};
__device__ __forceinline__ int token_of(const AttnArgs &a, int number) {
    return a.group == 1 ? number : (int)((uint32_t)number / (uint32_t)a.group);
}
template <int TILE>
__device__ __forceinline__ RowTile row_tile(const AttnArgs &a, int id, int lane, int block) {
    RowTile r;
    r.tile = a.row_tiles - 1 - id % a.row_tiles;      // the long rows of a causal mask first
    id /= a.row_tiles;
    r.hk = id % a.Hk;
    r.b = id / a.Hk;
    r.s = sequence(a, r.b);
    r.start = r.tile * TILE;
    r.rows = r.s.nq * a.group - r.start;              // (tq * group < 2^31)
    r.rows = r.rows < TILE ? r.rows : TILE;
    const int mine = block * 32 + (lane & 31);
    r.valid = mine < r.rows;
    const int number = r.start + (r.valid ? mine : r.rows - 1);
    r.t = token_of(a, number);
    r.g = number - r.t * a.group;
    r.head = r.hk * a.group + r.g;
    r.first = first_seen(a, r.s, r.t);
    r.last = last_seen(a, r.s, r.t);
    r.block_low = __builtin_amdgcn_readlane(r.first, 0);
    r.block_full = __builtin_amdgcn_readlane(r.first, 31);
    r.block_end = __builtin_amdgcn_readlane(r.last, 0);
    r.block_high = block * 32 < r.rows ? __builtin_amdgcn_readlane(r.last, 31) : -1;
    r.low = first_seen(a, r.s, token_of(a, r.start));
    r.high = last_seen(a, r.s, token_of(a, r.start + r.rows - 1));
    return r;
}
// lam of the lane's head, made by the whole wave for each head of the group.
__device__ __forceinline__ float row_weight(const AttnArgs &a, const RowTile &r, int lane) {
    float lam = 0.f;
    for (int k = 0; k < a.group; ++k) {
        const float w = weight_of(a.weight, r.hk * a.group + k, lane).lam;
        lam = k == r.g ? w : lam;
    }
    return lam;
}
// Scores of 32 keys from j0 for the lane's row, of keys that it does not see minus infinity.
template <int MAPS>
__device__ __forceinline__ void hide(const RowTile &r, int j0, int lane, v16f (&z)[MAPS]) {
    const int at = j0 + 4 * (lane >> 5) - r.first;
    const uint32_t span = (uint32_t)(r.last - r.first);
    const bool none = r.last < r.first;
#pragma unroll
    for (int e = 0; e < 16; ++e) {
        const bool seen = !none && (uint32_t)(at + 8 * (e / 4) + e % 4) <= span;
#pragma unroll
        for (int i = 0; i < MAPS; ++i) z[i][e] = seen ? z[i][e] : -__builtin_inff();
    }
}

}  // namespace
}  // namespace nmspmm
