// Device-side helpers of the attention kernels (gfx950 only): operands of the 32x32 matrix instructions, tiles in LDS, packed sequences.
//
// All products are formed as 32 x 32 tiles.  Lane l of a wave, r = l % 32 and h = l / 32, holds of an operand the eight numbers
// (r, k = 8h .. 8h + 7) of a step of 16, and of a result the column r and the rows 8 (i / 4) + 4 h + i % 4, i = 0 .. 15.  The numbers
// i = 8s .. 8s + 7 of a result are therefore an operand of step s of the next product without any exchange between lanes, whose
// other operand takes its k in the same order: rows 16 s + 4 h + 0 .. 3 and 16 s + 8 + 4 h + 0 .. 3 of a tile ("columns" below).
#pragma once
#include <type_traits>

#include "attn_kernels.h"
#include "attn_prompt_plan.h"
#include "lm_device.h"

typedef float v16f __attribute__((ext_vector_type(16)));
typedef float v8f __attribute__((ext_vector_type(8)));
typedef short v4s __attribute__((ext_vector_type(4)));

template <class E>
struct Operand {
    typedef E type __attribute__((ext_vector_type(8)));
};

__device__ __forceinline__ v16f multiply(Operand<__bf16>::type a, Operand<__bf16>::type b, v16f c)
{
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
}
__device__ __forceinline__ v16f multiply(Operand<_Float16>::type a, Operand<_Float16>::type b, v16f c)
{
    return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0);
}
// binary32: eight products of two steps each, which take k = i of both halves in step i.
__device__ __forceinline__ v16f multiply(v8f a, v8f b, v16f c)
{
#pragma unroll
    for (int i = 0; i < 8; ++i) c = __builtin_amdgcn_mfma_f32_32x32x2f32(a[i], b[i], c, 0, 0, 0);
    return c;
}

// Numbers 8s .. 8s + 7 of a result as an operand, rounded to the type: a product's operands have its inputs' type.
template <class E>
__device__ __forceinline__ typename Operand<E>::type operand_of(const v16f &c, int s)
{
    v8f part;
#pragma unroll
    for (int i = 0; i < 8; ++i) part[i] = c[8 * s + i];
    return __builtin_convertvector(part, typename Operand<E>::type);
}

// ---- tiles in LDS: rows of HD elements, their 16-byte units exchanged within a row by a function of the row's number, so that
// neither 16 lanes that read the same unit of 16 rows nor four rows of 64 bytes that are read as columns meet in a bank.
template <class E, int HD>
struct Tile {
    static constexpr int PER = 16 / (int)sizeof(E);          // elements of a unit
    static constexpr int UNITS = HD / PER;
    static __device__ __forceinline__ int place(int row, int unit)
    {
        const int f = UNITS >= 16 ? (row & 3) << 2 | (row >> 2 & 3) : (row >> 1 & 1) << 2 | (row >> 2 & 3);
        return row * HD + (unit ^ f) * PER;
    }
    // (row r, k = 16 s + 8 h .. + 7)
    static __device__ __forceinline__ typename Operand<E>::type row_operand(const E *t, int row, int s, int h)
    {
        typename Operand<E>::type v;
        if constexpr (sizeof(E) == 2) {
            v = *reinterpret_cast<const typename Operand<E>::type *>(t + place(row, 2 * s + h));
        } else {
            const v4f lo = *reinterpret_cast<const v4f *>(t + place(row, 4 * s + 2 * h));
            const v4f hi = *reinterpret_cast<const v4f *>(t + place(row, 4 * s + 2 * h + 1));
            v = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
        }
        return v;
    }
    // (column d0 + r, rows k0 + 4 h + 0 .. 3 and k0 + 8 + 4 h + 0 .. 3): 16 lanes read four rows of 16 elements and exchange them
    static __device__ __forceinline__ typename Operand<E>::type column_operand(const E *t, int k0, int d0, int lane)
    {
        typename Operand<E>::type v;
        if constexpr (sizeof(E) == 2) {
            const int row = k0 + (lane >> 5) * 4 + (lane >> 2 & 3);
            const int unit = d0 / 8 + (lane >> 4 & 1) * 2 + (lane >> 1 & 1), in = (lane & 1) * 4;
            typedef __attribute__((address_space(3))) v4s *lds;
            union {
                v4s half[2];
                typename Operand<E>::type all;
            } u;
            u.half[0] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds)(t + place(row, unit) + in));
            u.half[1] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds)(t + place(row + 8, unit) + in));
            v = u.all;
        } else {
            const int d = d0 + (lane & 31), row = k0 + (lane >> 5) * 4;
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = t[place(row + i % 4 + i / 4 * 8, d / 4) + d % 4];
        }
        return v;
    }
};

// Lanes of one wave read what others of it wrote to LDS: they do so in order, and the compiler is not to change it.
__device__ __forceinline__ void wave_order()
{
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
}

// The wave's number within its workgroup, known to the compiler to be the same for all lanes.
__device__ __forceinline__ int wave_number() { return __builtin_amdgcn_readfirstlane(threadIdx.x >> 6); }

// Rows of a tile on their way from memory to LDS: 16 bytes at a time, side by side in a row for lanes side by side.
template <class E, int HD, int ROWS, int THREADS = 256>
struct Mover {
    typedef Tile<E, HD> T;
    static constexpr int PIECES = ROWS * T::UNITS / THREADS, STEP = THREADS / T::UNITS;
    v4u at[PIECES];
    // Rows first .. first + ROWS - 1 of `p`; the last before `end` again from there on (what they are worth, the caller leaves out), and
    // the first unit again past the elements of a head (their products meet zeros or are not stored): no load is behind a branch.
    // Whole tiles take one offset for all lanes' pieces and addresses that the scalar unit forms.
    __device__ __forceinline__ void fetch(const E *p, int64_t stride, int first, int end, int dim)
    {
        int u = threadIdx.x % T::UNITS;
        const int row = threadIdx.x / T::UNITS;
        u = u * T::PER < dim ? u * T::PER : 0;
        if (first + ROWS <= end && stride <= 1 << 24) {
            const uint32_t off = ((uint32_t)row * (uint32_t)stride + u) * (uint32_t)sizeof(E);
            const char *from = reinterpret_cast<const char *>(p + first * stride);
#pragma unroll
            for (int i = 0; i < PIECES; ++i) at[i] = *reinterpret_cast<const v4u *>(from + i * STEP * stride * (int)sizeof(E) + off);
        } else {
#pragma unroll
            for (int i = 0; i < PIECES; ++i) {
                const int j = first + row + STEP * i;
                at[i] = *reinterpret_cast<const v4u *>(p + u + (j < end ? j : end - 1) * stride);
            }
        }
    }
    __device__ __forceinline__ void put(E *t) const
    {
        const int u = threadIdx.x % T::UNITS, row = threadIdx.x / T::UNITS;
        E *const to = t + T::place(row, u);
#pragma unroll
        for (int i = 0; i < PIECES; ++i)
            // (the exchange of units goes by the row's number modulo 16)
            *reinterpret_cast<v4u *>(STEP % 16 == 0 ? to + STEP * i * HD : t + T::place(row + STEP * i, u)) = at[i];
    }
};

// Tiles on their way from memory to LDS: start() sends for one, finish() has it there (for this wave; a barrier makes it everyone's).
// DIRECT: straight into LDS, without registers and stores: 64 lanes of a wave fill 1 KB of a tile side by side, so a lane fetches the
// unit that belongs in its place.  The tile has to be free from start() on; else from finish() on.
// (The loads are instructions the compiler does not know of.  They have no registers for it to use early, what it waits for itself
// it waits for no less long, and finish() waits for all.)
template <class E, int HD, int ROWS, bool DIRECT, int THREADS = 256>
struct Feed {
    typedef Tile<E, HD> T;
    static constexpr int PIECES = ROWS * T::UNITS / THREADS, STEP = THREADS / T::UNITS;
    static_assert(!DIRECT || STEP % 16 == 0, "the exchange of units goes by the row's number modulo 16");
    Mover<E, HD, ROWS, THREADS> mover;
    __device__ __forceinline__ void start(E *t, const E *p, int64_t stride, int first, int end, int dim)
    {
        if constexpr (!DIRECT) {
            mover.fetch(p, stride, first, end, dim);
            return;
        }
        const int row = threadIdx.x / T::UNITS, unit = T::place(row, threadIdx.x % T::UNITS) - row * HD, u = unit < dim ? unit : 0;
        const uint32_t base = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char *)t + wave_number() * 1024;
        if (first + ROWS <= end && stride <= 1 << 24) {
            const uint32_t off = ((uint32_t)row * (uint32_t)stride + u) * (uint32_t)sizeof(E);
            const char *from = reinterpret_cast<const char *>(p + first * stride);
#pragma unroll
            for (int i = 0; i < PIECES; ++i)
                asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"(base + i * THREADS * 16), "v"(off),
                             "s"(from + i * STEP * stride * (int)sizeof(E))
                             : "memory", "m0");
        } else {
#pragma unroll
            for (int i = 0; i < PIECES; ++i) {
                const int j = first + row + STEP * i;
                asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off" ::"s"(base + i * THREADS * 16),
                             "v"(p + u + (j < end ? j : end - 1) * stride)
                             : "memory", "m0");
            }
        }
    }
    __device__ __forceinline__ void finish(E *t)
    {
        if constexpr (DIRECT) asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        else mover.put(t);
    }
};

// Keeps the compiler from computing a rarely taken branch's selections always.
__device__ __forceinline__ void stay_a_branch() { asm volatile(""); }

// Heads of up to 64, 96 and 128 elements have kernels of their own (WIDTH); rows of a tile have 64 or 128.
template <int WIDTH>
constexpr int kRow = WIDTH == 64 ? 64 : 128;

// Schedule of the products just written: FIRST of their READS loads from LDS before the first of MANY products, the others one after each, so
// that a product does not wait for its own load.
template <int READS, int MANY, int FIRST>
__device__ __forceinline__ void ahead()
{
    __builtin_amdgcn_sched_group_barrier(0x100, FIRST, 0);
    constexpr int EACH = (READS - FIRST + MANY - 1) / MANY;
#pragma unroll
    for (int i = 0; i < MANY; ++i) {
        __builtin_amdgcn_sched_group_barrier(0x8, 1, 0);
        if (EACH > 0 && FIRST + i * EACH < READS) __builtin_amdgcn_sched_group_barrier(0x100, EACH, 0);
    }
}

__device__ __forceinline__ v16f zeros()
{
    v16f z;
#pragma unroll
    for (int i = 0; i < 16; ++i) z[i] = 0.0f;
    return z;
}

// Adds up what `parts` waves hold, in their order: wave w of them leaves its numbers in LDS, the first adds and keeps the sum.
// All waves of the workgroup take part; `of` numbers the groups of waves, `part` the wave within its group.
template <int DT>
__device__ __forceinline__ void join(v16f (&o)[DT], float *room, int of, int groups, int part, int parts, int lane)
{
    if (parts == 1) return;
    __syncthreads();
    if (part > 0) {
        float *mine = room + (int64_t)((part - 1) * groups + of) * DT * 1024 + lane;
#pragma unroll
        for (int d = 0; d < DT; ++d)
#pragma unroll
            for (int i = 0; i < 16; ++i) mine[(d * 16 + i) * 64] = o[d][i];
    }
    __syncthreads();
    if (part > 0) return;
    for (int p = 0; p < parts - 1; ++p) {
        const float *its = room + (int64_t)(p * groups + of) * DT * 1024 + lane;
#pragma unroll
        for (int d = 0; d < DT; ++d)
#pragma unroll
            for (int i = 0; i < 16; ++i) o[d][i] += its[(d * 16 + i) * 64];
    }
}

constexpr int most(int a, int b) { return a > b ? a : b; }

// One number for both lanes of a column.
__device__ __forceinline__ float both_max(float v)
{
    const auto s = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return __builtin_elementwise_maximum(__uint_as_float(s[0]), __uint_as_float(s[1]));
}
__device__ __forceinline__ float both_sum(float v)
{
    const auto s = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return __uint_as_float(s[0]) + __uint_as_float(s[1]);
}

__device__ __forceinline__ bool is_finite(float v) { return (__float_as_uint(v) & 0x7f800000u) != 0x7f800000u; }

// The eight elements from element 8u of a head (zeros past its last and where there is no row), in the order of memory.
template <class E>
__device__ __forceinline__ typename Operand<E>::type load_unit8(const E *row, int u, int dim, bool there)
{
    typename Operand<E>::type v = {};
    if (there && u * 8 < dim) {
        if constexpr (sizeof(E) == 2) {
            v = *reinterpret_cast<const typename Operand<E>::type *>(row + u * 8);
        } else {
            const v4f lo = *reinterpret_cast<const v4f *>(row + u * 8), hi = *reinterpret_cast<const v4f *>(row + u * 8 + 4);
            v = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
        }
    }
    return v;
}

// Operands of 32 keys straight from memory, for a wave that shares its keys with no other.  binary32 alone: a column's elements are whole
// words of a lane.  Keys from `end` on are the last one again, elements past a head's its first (as a Mover's).
template <int WIDTH>
struct RowOperands {
    v8f at[WIDTH / 16];
    __device__ __forceinline__ void fetch(const float *p, int64_t stride, int first, int end, int dim, int lane)
    {
        const int j = first + (lane & 31), h = lane >> 5;
        const float *row = p + (j < end ? j : end - 1) * stride;
#pragma unroll
        for (int i = 0; i < WIDTH / 16; ++i) {
            const float *from = row + ((2 * i + h) * 8 < dim ? (2 * i + h) * 8 : 0);
            at[i] = __builtin_shufflevector(*reinterpret_cast<const v4f *>(from), *reinterpret_cast<const v4f *>(from + 4), 0, 1, 2, 3, 4, 5, 6, 7);
        }
    }
};
template <int WIDTH>
struct ColumnOperands {
    v8f at[2][WIDTH / 32];
    __device__ __forceinline__ void fetch(const float *p, int64_t stride, int first, int end, int dim, int lane)
    {
        const int r = lane & 31, h = lane >> 5;
        const bool whole = first + 32 <= end && stride <= 1 << 24;
        const char *from = reinterpret_cast<const char *>(p + first * stride);
#pragma unroll
        for (int d = 0; d < WIDTH / 32; ++d) {
            const int u = d * 32 + r < dim ? d * 32 + r : 0;
            const uint32_t off = ((uint32_t)(4 * h) * (uint32_t)stride + u) * 4;
#pragma unroll
            for (int n = 0; n < 16; ++n) {
                const int key = n / 8 * 16 + n / 4 % 2 * 8 + n % 4, j = first + 4 * h + key;
                at[n / 8][d][n % 8] = whole ? *reinterpret_cast<const float *>(from + key * stride * 4 + off) : p[(j < end ? j : end - 1) * stride + u];
            }
        }
    }
};

// ---- packed sequences ---------------------------------------------------------------------------
//
// How they number their tiles: attn_prompt_plan.h.
struct Sequence {
    int at, q0, q_len, k0, k_len;            // at: the tile's first row within the sequence; negative: no tile
};

__device__ __forceinline__ int clamped(int v, int most) { return v < 0 ? 0 : v > most ? most : v; }

// All 64 lanes take part, with the same arguments: the last sequence whose first tile (or, with tile 0, first row) is not behind `number`;
// negative if there is none.
__device__ __forceinline__ int find_sequence(const int32_t *starts, int rows, int sequences, int tile, int number)
{
    const int lane = threadIdx.x & 63;
    int lo = 0, n = sequences;
    while (true) {
        const int step = (n + 63) / 64, s = lane * step < n ? lo + lane * step : lo, start = clamped(starts[s], rows);
        const int count = __popcll(__ballot(lane * step < n && (tile ? attn_first_tile(start, tile, s) : start) <= number));
        if (count == 0) return -1;
        lo += (count - 1) * step;
        n = n - (count - 1) * step < step ? n - (count - 1) * step : step;
        if (n <= 1) return __builtin_amdgcn_readfirstlane(lo);
    }
}

// by_keys: the tiles are of keys.
__device__ __forceinline__ Sequence tile_of(const int32_t *q_starts, const int32_t *k_starts, int q_rows, int k_rows, int sequences,
                                            bool by_keys, int tile, int number)
{
    Sequence s = {-1, 0, q_rows, 0, k_rows};
    if (!q_starts) {
        s.at = number * tile;
    } else {
        const int rows = by_keys ? k_rows : q_rows;
        const int32_t *starts = by_keys ? k_starts : q_starts;
        const int i = find_sequence(starts, rows, sequences, tile, number);
        if (i < 0) return s;
        s.q0 = clamped(q_starts[i], q_rows);
        s.q_len = clamped(q_starts[i + 1], q_rows) - s.q0;
        s.k0 = clamped(k_starts[i], k_rows);
        s.k_len = clamped(k_starts[i + 1], k_rows) - s.k0;
        if (s.q_len < 0) s.q_len = 0;
        if (s.k_len < 0) s.k_len = 0;
        s.at = (number - attn_first_tile(by_keys ? s.k0 : s.q0, tile, i)) * tile;
    }
    if (s.at >= (by_keys ? s.k_len : s.q_len)) s.at = -1;
    return s;
}

// Number of keys that row i of a sequence sees.
__device__ __forceinline__ int visible(const Sequence &s, int causal, int i)
{
    const int n = causal ? i + s.k_len - s.q_len + 1 : s.k_len;
    return n < 0 ? 0 : n > s.k_len ? s.k_len : n;
}

constexpr float kLog2e = 1.44269504088896340736f, kLn2 = 0.69314718055994530942f;
// A softmax's reference before its first key: below every score, and finite, so that differences with it are numbers.
constexpr float kNoKey = -3.0e38f;
// The reference may lag behind the largest score by kLag (to base 2): up to there sums and operands lose nothing, and raising it takes 64
// products a lane.  In float16, where an operand below 2^-14 loses digits and one of 2^-25 is zero, probabilities enter sums and products times
// 2^kSumLift, of which results are free, and the reference lags less, so that they stay below 2^15: a probability has all its digits from 2^-27 of
// its row's largest on, and 2^21 keys that vanish are at most 2^-17 of a row.
template <class E>
constexpr bool kLifted = std::is_same<E, _Float16>::value;
template <class E>
constexpr float kLag = kLifted<E> ? 2.0f : 8.0f;
template <class E>
constexpr float kSumLift = kLifted<E> ? 13.0f : 0.0f;
template <class E>
constexpr float kSumDrop = kLifted<E> ? 0x1p-13f : 1.0f;

// ---- a block of keys ----------------------------------------------------------------------------------
//
// 32 KT keys for the 32 rows of a wave: running maximum m and sum l (of the scores times c, to base 2) of the lane's row and the
// transposed sums o, both times 2^kSumLift.  key(n, i) and value(n, half, d) are the operands of 32 keys n, `hide` puts -inf in the place of scores that are not seen.
template <class E, int WIDTH, int KT, class Key, class Value, class Hide>
__device__ __forceinline__ void attend_to(Key key, Value value, const typename Operand<E>::type (&q)[WIDTH / 16], float c, float &m, float &l,
                                          v16f (&o)[WIDTH / 32], Hide hide)
{
    v16f x[KT];
#pragma unroll
    for (int n = 0; n < KT; ++n) {
        x[n] = zeros();
#pragma unroll
        for (int i = 0; i < WIDTH / 16; ++i) x[n] = multiply(key(n, i), q[i], x[n]);
    }
    if (sizeof(E) == 2) ahead<KT * WIDTH / 16, KT * WIDTH / 16, 6>();        // (2 % of a long prompt's time)
    hide(x);
    float most = x[0][0];
#pragma unroll
    for (int n = 0; n < KT; ++n)
#pragma unroll
        for (int i = 0; i < 16; ++i) most = __builtin_elementwise_maximum(most, x[n][i]);
    most = both_max(most) * c;
    if (__any(most > m + kLag<E>)) {
        const float next = most > m ? most : m, f = __builtin_amdgcn_exp2f(m - next);
        m = next;
        l *= f;
#pragma unroll
        for (int d = 0; d < WIDTH / 32; ++d)
#pragma unroll
            for (int i = 0; i < 16; ++i) o[d][i] *= f;
    }
    const float ref = kLifted<E> ? kSumLift<E> - m : -m;
#pragma unroll
    for (int n = 0; n < KT; ++n)
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            x[n][i] = __builtin_amdgcn_exp2f(__builtin_fmaf(x[n][i], c, ref));
            l += x[n][i];
        }
#pragma unroll
    for (int n = 0; n < KT; ++n)
#pragma unroll
        for (int half = 0; half < 2; ++half) {
            const typename Operand<E>::type p = operand_of<E>(x[n], half);
#pragma unroll
            for (int d = 0; d < WIDTH / 32; ++d) o[d] = multiply(value(n, half, d), p, o[d]);
        }
}
// The same from row `in` of the tiles kt and vt on.
template <class E, int WIDTH, int KT, class Hide>
__device__ __forceinline__ void attend(const E *kt, const E *vt, int in, const typename Operand<E>::type (&q)[WIDTH / 16], float c, float &m, float &l,
                                       v16f (&o)[WIDTH / 32], int lane, Hide hide)
{
    typedef Tile<E, kRow<WIDTH>> T;
    const int r = lane & 31, h = lane >> 5;
    attend_to<E, WIDTH, KT>([=](int n, int i) { return T::row_operand(kt, in + n * 32 + r, i, h); },
                            [=](int n, int half, int d) { return T::column_operand(vt, in + n * 32 + half * 16, d * 32, lane); }, q, c, m, l, o, hide);
}

// ---- rows that are not finite ---------------------------------------------------------------------
//
// A key that a row does not see counts for nothing, but in a product of whole tiles its zero meets its value, and zero times an infinity or
// NaN is NaN; and sums of values near the end of binary32 may pass it on the way.  Most rows that are not finite are so because of what they see, and an
// infinity or NaN early in a sequence is seen by all rows after it, so a row is looked at in three steps:
//   - the sum of its softmax is not finite: it sees a score that is NaN or plus infinity (hidden keys have no part in the sum), and nothing of it is finite;
//   - each of its elements that is not finite sees a value that is not: the sum of those, infinity or NaN, is the element;
//   - else the row is formed again from the keys it sees alone, by one wave: 2 to 4 ms for a row of 16384 keys.  In a causal prompt those are at most 94 rows
//     a head for each value that is not finite (the ones before it in its tile of 64 keys and beside those in their 32 rows), and the rows whose sums pass
//     binary32.
// Keys: `int count()`, `int64_t place(j)` of key j, negative if it is not seen, `const E *key(place)`, `const E *value(place)`.

// Elements of a head, bit d % 64 of word d / 64: NaN, and infinities.
struct Spoilt {
    uint64_t nan[2], inf[2];
    __device__ __forceinline__ bool explained_by(const Spoilt &v) const
    {
        return !((nan[0] & ~v.nan[0]) | (nan[1] & ~v.nan[1]) | (inf[0] & ~v.inf[0]) | (inf[1] & ~v.inf[1]));
    }
};
// Of the elements lane and lane + 64 of all lanes.
__device__ __forceinline__ Spoilt spoilt_of(float y0, float y1)
{
    return {{__ballot(y0 != y0), __ballot(y1 != y1)}, {__ballot(__builtin_fabsf(y0) == INFINITY), __ballot(__builtin_fabsf(y1) == INFINITY)}};
}

// Lane i's number, known to be the same for all lanes.
__device__ __forceinline__ float lanes_number(float v, int i) { return __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(v), i)); }
__device__ __forceinline__ int64_t lanes_number(int64_t v, int i)
{
    return (int64_t)__builtin_amdgcn_readlane((int)(v >> 32), i) << 32 | (uint32_t)__builtin_amdgcn_readlane((int)v, i);
}

// The keys at a wave's 64 places (negative: not seen), kAtOnce at a time, while take(places at(i), i = 0 .. kAtOnce - 1, bits of those that are seen) says so.
// The place of one that is seen stands for one that is not.
constexpr int kAtOnce = 8;
template <class Take>
__device__ __forceinline__ void seen_keys(int64_t place, Take take)
{
    const uint64_t seen = __ballot(place >= 0);
    const int other = __ffsll((unsigned long long)seen) - 1;
#pragma unroll 1
    for (int i0 = 0; i0 < 64; i0 += kAtOnce) {
        const uint32_t mask = (uint32_t)(seen >> i0) & ((1u << kAtOnce) - 1);
        if (mask && !take([&](int i) { return lanes_number(place, mask >> i & 1 ? i0 + i : other); }, mask)) return;
    }
}
// Elements lane and lane + 64 of kAtOnce vectors, zeros past a head's last.
template <class E>
struct AtOnce {
    float low[kAtOnce], high[kAtOnce];
    template <class Vector>
    __device__ __forceinline__ void load(Vector vector, int dim)
    {
        const int lane = threadIdx.x & 63;
#pragma unroll
        for (int i = 0; i < kAtOnce; ++i) {
            const E *p = vector(i);
            low[i] = (float)p[lane < dim ? lane : 0], high[i] = (float)p[lane + 64 < dim ? lane + 64 : 0];
        }
#pragma unroll
        for (int i = 0; i < kAtOnce; ++i) low[i] = lane < dim ? low[i] : 0.0f, high[i] = lane + 64 < dim ? high[i] : 0.0f;
    }
};

// Adds to y (elements lane and lane + 64) what is not finite in the values of the keys from `from` on, until that explains `wanted`.  All lanes take part.
template <class E, class Keys>
__device__ __forceinline__ Spoilt add_spoilt(const Keys &keys, int from, int dim, const Spoilt &wanted, float (&y)[2])
{
    const int lane = threadIdx.x & 63, count = keys.count();
    Spoilt found = spoilt_of(y[0], y[1]);
#pragma unroll 1
    for (int j0 = from; j0 < count && !wanted.explained_by(found); j0 += 64) {
        seen_keys(j0 + lane < count ? keys.place(j0 + lane) : -1, [&](auto at, uint32_t) {
            AtOnce<E> v;
            v.load([&](int i) { return keys.value(at(i)); }, dim);
#pragma unroll
            for (int i = 0; i < kAtOnce; ++i) {
                y[0] += is_finite(v.low[i]) ? 0.0f : v.low[i];
                y[1] += is_finite(v.high[i]) ? 0.0f : v.high[i];
            }
            return true;
        });
        found = spoilt_of(y[0], y[1]);
    }
    return found;
}
// Do the values `z` that are not finite stand for all elements that are not?
__device__ __forceinline__ bool stands_for(const float (&z)[2], const Spoilt &its)
{
    const int lane = threadIdx.x & 63;
    return !__any(((its.nan[0] | its.inf[0]) >> lane & 1 && is_finite(z[0])) || ((its.nan[1] | its.inf[1]) >> lane & 1 && is_finite(z[1])));
}

// Is there a NaN in the keys?
template <class E, class Keys>
__device__ __forceinline__ bool nan_among(const Keys &keys, int dim)
{
    const int lane = threadIdx.x & 63, count = keys.count();
    bool found = false;
#pragma unroll 1
    for (int j0 = 0; j0 < count && !__any(found); j0 += 64)
        seen_keys(j0 + lane < count ? keys.place(j0 + lane) : -1, [&](auto at, uint32_t) {
            AtOnce<E> k;
            k.load([&](int i) { return keys.key(at(i)); }, dim);
#pragma unroll
            for (int i = 0; i < kAtOnce; ++i) found |= k.low[i] != k.low[i] || k.high[i] != k.high[i];
            return true;
        });
    return __any(found);
}

// Which of a wave's `rows` (bit r: row r) have to be formed again.  row_of(r, y): the row's elements lane and lane + 64; keys_of(r): its keys, of which
// all of these rows see the first `common`.  Of the other rows put(r, y) stores those in whose place there is something else.
template <class E, class RowOf, class KeysOf, class Put>
__device__ __forceinline__ uint32_t rows_to_form(uint32_t rows, int dim, int common, RowOf row_of, KeysOf keys_of, Put put)
{
    uint32_t again = 0;
    Spoilt wanted = {{0, 0}, {0, 0}};
    for (uint32_t left = rows; left; left &= left - 1) {
        float y[2];
        row_of(__ffs(left) - 1, y);
        const Spoilt its = spoilt_of(y[0], y[1]);
#pragma unroll
        for (int e = 0; e < 2; ++e) wanted.nan[e] |= its.nan[e], wanted.inf[e] |= its.inf[e];
    }
    auto shared = keys_of(__ffs(rows) - 1);
    shared.n = common;
    float sum[2] = {0.0f, 0.0f};
    const Spoilt found = add_spoilt<E>(shared, 0, dim, wanted, sum);
    for (uint32_t left = rows; left; left &= left - 1) {
        const int i = __ffs(left) - 1;
        float y[2], z[2] = {sum[0], sum[1]};
        row_of(i, y);
        const Spoilt its = spoilt_of(y[0], y[1]);
        if (its.explained_by(found)) continue;
        add_spoilt<E>(keys_of(i), common, dim, {{~0ull, ~0ull}, {0, 0}}, z);
        if (!stands_for(z, its)) {
            again |= 1u << i;
            continue;
        }
#pragma unroll
        for (int e = 0; e < 2; ++e) y[e] = is_finite(z[e]) ? y[e] : z[e];
        put(i, y);
    }
    return again;
}

// Leaves the normed row in o (elements lane, lane + 64 of it) and returns the logarithm to base 2 of its sum.  One pass over the keys; o is a
// mean of the values so far at any time, so no sum passes the largest of them.
template <class E, class Keys>
__device__ __forceinline__ float row_again(const E *q, int dim, float c, const Keys &keys, float o[2])
{
    const int lane = threadIdx.x & 63, count = keys.count();
    const float q0 = lane < dim ? (float)q[lane] : 0.0f, q1 = lane + 64 < dim ? (float)q[lane + 64] : 0.0f;
    float m = kNoKey, l = 0.0f;
    o[0] = o[1] = 0.0f;
#pragma unroll 1
    for (int j0 = 0; j0 < count && m < INFINITY; j0 += 64)
        seen_keys(j0 + lane < count ? keys.place(j0 + lane) : -1, [&](auto at, uint32_t mask) {
            AtOnce<E> k, v;
            k.load([&](int i) { return keys.key(at(i)); }, dim);
            v.load([&](int i) { return keys.value(at(i)); }, dim);
            float s[kAtOnce], top = m, sum = 0.0f;
#pragma unroll
            for (int i = 0; i < kAtOnce; ++i) s[i] = __builtin_fmaf(q0, k.low[i], q1 * k.high[i]);
#pragma unroll
            for (int off = 32; off > 0; off >>= 1)
#pragma unroll
                for (int i = 0; i < kAtOnce; ++i) s[i] += __shfl_xor(s[i], off);
#pragma unroll
            for (int i = 0; i < kAtOnce; ++i) {
                s[i] = mask >> i & 1 ? s[i] * c : -INFINITY;
                top = __builtin_elementwise_maximum(top, s[i]);
            }
            const float before = l * __builtin_amdgcn_exp2f(m - top);
#pragma unroll
            for (int i = 0; i < kAtOnce; ++i) s[i] = __builtin_amdgcn_exp2f(s[i] - top), sum += s[i];
            m = top;
            l = before + sum;
            if (!(m < INFINITY)) return false;
            if (l == 0.0f) return true;                          // (scores of minus infinity alone)
            const float by = 1.0f / l;
            o[0] *= before * by, o[1] *= before * by;
#pragma unroll
            for (int i = 0; i < kAtOnce; ++i) {
                o[0] = mask >> i & 1 ? __builtin_fmaf(s[i] * by, v.low[i], o[0]) : o[0];
                o[1] = mask >> i & 1 ? __builtin_fmaf(s[i] * by, v.high[i], o[1]) : o[1];
            }
            return true;
        });
    // (a score of NaN or plus infinity: nothing of the row is finite; no sum: neither)
    if (!(m < INFINITY) || l == 0.0f) o[0] = o[1] = __builtin_nanf("");
    return m + __builtin_amdgcn_logf(l);
}
