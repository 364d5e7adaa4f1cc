// The 4-bit container (layout in include/mom.h) and the warp-level product on it.
//
// A warp multiplies 16 rows of W by up to 8 tokens per mma.sync m16n8k16, W as the A operand.  The container holds a 16 x 128
// tile as two times 512 consecutive bytes in the order of the operand fragments: lane 4 g + t owns, of rows g and g + 8, columns
// 4 t .. 4 t + 3 and 16 + 4 t .. 19 + 4 t of each stretch of 32 columns: the order in which tcgen05.st.16x256b lays two blocks of 16
// columns into tensor memory.  For mma.sync the contraction index may be permuted freely as long as both operands agree: the
// lane's eight columns are split over two MMAs (four each), and x is kept with the lane's eight entries side by side
// (place_of), one 16-byte load.
// Codes become operand entries by bit operations: 0x4300 | q is 128 + q in bf16, 0x6400 | q is 1024 + q and 0x5400 | q << 4 is 64 + q in
// f16; subtracting that + zero is exact.  These operations are what bounds the products: of a tile's 1024 bytes a lane makes 64
// codes, by 56 (f16: 40) integer instructions at half rate and 32 subtractions.  The scale is not multiplied in (that would round each weight): MMAs sum code * x of
// one group, and the group's f32 sums are scaled when they are added up.
#pragma once

#include "serve_common.cuh"

namespace mom {

// Where column k of a row of activations stands in the order of the mma.sync operand: within its 32, four by four, the
// halves alternating.
__host__ __device__ constexpr int place_of(int k) { return (k & ~31) | ((k & 12) << 1) | ((k & 16) >> 2) | (k & 3); }

constexpr int W4_ROWS = 16, W4_COLS = 128, W4_TILE_BYTES = 1024;

struct W4Geometry {
    long long row_tiles, col_tiles, groups;
    size_t scales_at, zeros_at, matrix_bytes;
};

inline W4Geometry w4_geometry(const mom_w4_desc_t &d) {
    W4Geometry g;
    g.row_tiles = (d.rows + W4_ROWS - 1) / W4_ROWS;
    g.col_tiles = (d.cols + W4_COLS - 1) / W4_COLS;
    g.groups = d.group ? g.col_tiles * (W4_COLS / d.group) : 1;      // whole tiles of them
    g.scales_at = align_up((size_t)g.row_tiles * g.col_tiles * W4_TILE_BYTES, WS_ALIGN);
    g.zeros_at = align_up(g.scales_at + (size_t)g.row_tiles * g.groups * W4_ROWS * element_bytes(d.scale_dtype), WS_ALIGN);
    g.matrix_bytes = d.zeros ? align_up(g.zeros_at + (size_t)g.row_tiles * g.groups * W4_ROWS, WS_ALIGN) : g.zeros_at;
    return g;
}

mom_status_t check_w4_desc(const mom_w4_desc_t *d);

// One matrix of a container as the kernels see it.
struct W4View {
    const uint8_t *base;
    long long matrix_bytes;           // from matrix to matrix
    long long scales_at, zeros_at;
    int rows, cols, row_tiles, col_tiles, groups;
    int group_shift;                  // column -> group
    int scale_dtype, has_zeros;
};

inline W4View w4_view(const mom_w4_desc_t &d, const void *container) {
    const W4Geometry g = w4_geometry(d);
    W4View v;
    v.base = static_cast<const uint8_t *>(container);
    v.matrix_bytes = (long long)g.matrix_bytes;
    v.scales_at = (long long)g.scales_at;
    v.zeros_at = (long long)g.zeros_at;
    v.rows = (int)d.rows;
    v.cols = (int)d.cols;
    v.row_tiles = (int)g.row_tiles;
    v.col_tiles = (int)g.col_tiles;
    v.groups = (int)g.groups;
    v.group_shift = group_shift(d.group);
    v.scale_dtype = d.scale_dtype;
    v.has_zeros = d.zeros;
    return v;
}

// ---- device side ----------------------------------------------------------------------------

template <bool BF16>
__device__ __forceinline__ uint32_t sub2(uint32_t a, uint32_t b) {
    uint32_t r;
    if (BF16) asm("sub.rn.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    else asm("sub.rn.f16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    return r;
}

// What is subtracted from a row's entries, as pairs: the bias of the bits plus the zero.
template <bool BF16> struct Offset {
    uint32_t low, high;                        // of the codes in bits 0-3 of a half word; in bits 4-7 (f16 only)
    __device__ __forceinline__ void set(uint32_t zero) {
        const uint32_t z = zero | (zero << 16);
        low = (BF16 ? 0x43004300u : 0x64006400u) + z;
        high = 0x54005400u + (z << 4);
    }
};

// (a & mask) | bits in one instruction (two constants: left to itself the compiler takes two)
__device__ __forceinline__ uint32_t and_or(uint32_t a, uint32_t mask, uint32_t bits) {
    uint32_t r;
    asm("lop3.b32 %0, %1, %2, %3, 0xEA;" : "=r"(r) : "r"(a), "r"(mask), "r"(bits));
    return r;
}

// eight codes -> four operand pairs (columns 0 1, 2 3, 4 5, 6 7), exact integers code - zero
template <bool BF16>
__device__ __forceinline__ void unpack_codes(uint32_t w, const Offset<BF16> &o, uint32_t (&p)[4]) {
    if (BF16) {
#pragma unroll
        for (int i = 0; i < 4; ++i) p[i] = sub2<true>(and_or(w >> (4 * i), 0x000f000fu, 0x43004300u), o.low);
    } else {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const uint32_t v = w >> (8 * i);
            p[2 * i] = sub2<false>(and_or(v, 0x000f000fu, 0x64006400u), o.low);
            p[2 * i + 1] = sub2<false>(and_or(v, 0x00f000f0u, 0x54005400u), o.high);
        }
    }
}

template <bool BF16>
__device__ __forceinline__ void mma16816(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    if (BF16)
        asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                     : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
    else
        asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                     : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
// the same with C = 0
template <bool BF16>
__device__ __forceinline__ void mma16816_first(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    if (BF16)
        asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%10, %10, %10, %10};"
                     : "=f"(c[0]), "=f"(c[1]), "=f"(c[2]), "=f"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1), "f"(0.0f));
    else
        asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%10, %10, %10, %10};"
                     : "=f"(c[0]), "=f"(c[1]), "=f"(c[2]), "=f"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1), "f"(0.0f));
}

// ---- eight consecutive activations as token operand -------------------------------------------
// As loaded: 32, 16 or 8 bytes.
template <int DTYPE> struct Raw8 { uint32_t r[DTYPE == MOM_F32 ? 8 : DTYPE == MOM_E4M3 || DTYPE == MOM_INT8 ? 2 : 4]; };

// Columns k .. k + 7 of a row, zeros beyond `cols`.  wide: the row starts on a 16-byte
// boundary, so that whole groups of eight inside the row take 16-byte (8 bits: 8-byte) loads.
template <int DTYPE>
__device__ __forceinline__ Raw8<DTYPE> load_x8(const void *row, int k, int cols, bool wide) {
    using T = typename Element<DTYPE>::type;
    constexpr int WORDS = sizeof(Raw8<DTYPE>) / 4;
    Raw8<DTYPE> v;
#pragma unroll
    for (int i = 0; i < WORDS; ++i) v.r[i] = 0;
    if (k >= cols) return v;
    const T *p = static_cast<const T *>(row) + k;
    if (wide && k + 8 <= cols) {
        if (WORDS == 2) {
            const uint2 a = *reinterpret_cast<const uint2 *>(p);
            v.r[0] = a.x; v.r[1] = a.y;
        } else {
#pragma unroll
            for (int i = 0; i < WORDS / 4; ++i) {
                const uint4 a = reinterpret_cast<const uint4 *>(p)[i];
                v.r[4 * i] = a.x; v.r[4 * i + 1] = a.y; v.r[4 * i + 2] = a.z; v.r[4 * i + 3] = a.w;
            }
        }
        return v;
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        if (k + i >= cols) continue;
        if (sizeof(T) == 4) v.r[i * WORDS / 8] = reinterpret_cast<const uint32_t *>(p)[i];
        else if (sizeof(T) == 2) v.r[i * WORDS / 8] |= (uint32_t) reinterpret_cast<const uint16_t *>(p)[i] << (16 * (i & 1));
        else v.r[i * WORDS / 8] |= (uint32_t) reinterpret_cast<const uint8_t *>(p)[i] << (8 * (i & 3));
    }
    return v;
}

// f32 pair -> three bf16 pairs whose sum is the pair exactly: each term takes the leading 8 bits that are left (truncated, so that
// nothing overflows).  An infinity stays in the first term alone.
__device__ __forceinline__ void split_pair(float a, float b, uint32_t &t0, uint32_t &t1, uint32_t &t2) {
    const uint32_t ua = __float_as_uint(a), ub = __float_as_uint(b);
    t0 = __byte_perm(ua, ub, 0x7632);
    float ra = a - __uint_as_float(ua & 0xffff0000u), rb = b - __uint_as_float(ub & 0xffff0000u);
    if ((ua << 1) == 0xff000000u) ra = 0.0f;
    if ((ub << 1) == 0xff000000u) rb = 0.0f;
    const uint32_t va = __float_as_uint(ra), vb = __float_as_uint(rb);
    t1 = __byte_perm(va, vb, 0x7632);
    const float sa = ra - __uint_as_float(va & 0xffff0000u), sb = rb - __uint_as_float(vb & 0xffff0000u);
    t2 = __byte_perm(__float_as_uint(sa), __float_as_uint(sb), 0x7632);
}

// eight activations -> operand pairs, term by term
template <int DTYPE, int TERMS>
__device__ __forceinline__ void expand_x8(const Raw8<DTYPE> &v, uint32_t (&b)[TERMS][4]) {
    if constexpr (DTYPE == MOM_F32) {
#pragma unroll
        for (int i = 0; i < 4; ++i) split_pair(__uint_as_float(v.r[2 * i]), __uint_as_float(v.r[2 * i + 1]), b[0][i], b[1][i], b[2][i]);
    } else if constexpr (DTYPE == MOM_BF16 || DTYPE == MOM_F16) {
#pragma unroll
        for (int i = 0; i < 4; ++i) b[0][i] = v.r[i];
    } else if constexpr (DTYPE == MOM_E4M3) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const __half2_raw h = __nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)(v.r[i >> 1] >> (16 * (i & 1))), __NV_E4M3);
            b[0][i] = (uint32_t)h.x | ((uint32_t)h.y << 16);
        }
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) {                 // 0x6400 | u is 1024 + u in f16; u = code + 128
            const uint32_t u = v.r[i >> 1] ^ 0x80808080u;
            b[0][i] = sub2<false>(__byte_perm(u, 0x64646464u, (i & 1) ? 0x4342 : 0x4140), 0x64806480u);
        }
    }
}

// `tiles` tiles dealt to `warps` warps in even stretches: warp w's is [first, end).
struct Stretch {
    int first, end;
    __device__ __forceinline__ Stretch(int tiles, int warps, int w) : first(tiles * w / warps), end(tiles * (w + 1) / warps) {}
};
// the warp whose stretch holds tile `at`
__device__ __forceinline__ int stretch_of(int tiles, int warps, int at) {
    int w = at * warps / tiles;
    while (Stretch(tiles, warps, w).end <= at) ++w;
    return w;
}

// ---- a warp's stream of tiles ------------------------------------------------------------------
// Tiles travel from global memory through a ring in shared memory that belongs to one warp: cp.async (16 bytes a lane), so
// that several are on their way while one is multiplied, without registers and without barriers between
// warps.  A slot takes two neighbouring tiles of a row (the bookkeeping costs as much for one) with the scales and zeros of
// their groups.

__device__ __forceinline__ void copy16(uint32_t dst, const void *src) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
}

// How a slot is laid out: codes of two tiles, then the scales and the zeros of their groups.
struct SlotLayout {
    int tile_groups;            // groups of a tile: 1, 2 or 4
    int group_step;             // groups from tile to tile (0: one scale per row)
    int scale_bytes;            // 16 scales of a group
    int zeros_at, bytes;
};
__host__ __device__ inline SlotLayout slot_layout(const W4View &w) {
    SlotLayout s;
    s.tile_groups = w.group_shift >= 7 ? 1 : W4_COLS >> w.group_shift;
    s.group_step = w.group_shift == 31 ? 0 : s.tile_groups;
    s.scale_bytes = w.scale_dtype == MOM_F32 ? 64 : 32;
    s.zeros_at = 2 * W4_TILE_BYTES + 2 * s.tile_groups * s.scale_bytes;
    s.bytes = s.zeros_at + (w.has_zeros ? 2 * s.tile_groups * 16 : 0);
    return s;
}
constexpr int MAX_SLOT_BYTES = 2 * W4_TILE_BYTES + 8 * 64 + 8 * 16;

// What a lane copies for the next slot: its 16 bytes of the codes' four parts and, if it has a part in them, of the scales and
// zeros.  BOTH: the slot takes one tile of each of two matrices of the same geometry, else two neighbouring tiles of a row.
template <bool BOTH>
struct TileSource {
    const uint8_t *codes, *other, *scales, *zeros;
};

template <int SLOTS>
struct TileRing {
    SlotLayout slot;
    uint32_t base, head, tail, end;   // shared address of the ring (this lane's 16 bytes); next slot to fill, next slot to use, size (bytes)
    int my_tile, my_group;            // whose scales the lane brings (my_tile > 1: none): the slot's tile and its group
    int my_zero;                      // and whose zeros (lane / tile_groups; > 1: none)

    __device__ __forceinline__ TileRing(uint32_t at, const W4View &w) : slot(slot_layout(w)), head(0), tail(0) {
        const int lane = threadIdx.x & 31, per = slot.scale_bytes / 16;
        base = at + lane * 16;
        end = SLOTS * slot.bytes;
        my_group = lane / per % slot.tile_groups;
        my_tile = lane / per / slot.tile_groups;
        my_zero = w.has_zeros ? lane / slot.tile_groups : 2;
    }

    // row tile rt of the matrix at m, from its tile kt on
    template <bool BOTH>
    __device__ __forceinline__ TileSource<BOTH> source(const W4View &w, const uint8_t *m, int rt, int kt) const {
        const int lane = threadIdx.x & 31, per = slot.scale_bytes / 16;
        const long long group = (long long)rt * w.groups + kt * slot.group_step;
        TileSource<BOTH> s;
        s.codes = m + ((long long)rt * w.col_tiles + kt) * W4_TILE_BYTES + lane * 16;
        s.other = nullptr;
        s.scales = m + w.scales_at + (group + my_group + (BOTH ? 0 : my_tile * slot.group_step)) * slot.scale_bytes + lane % per * 16;
        s.zeros = m + w.zeros_at + (group + lane - my_zero * slot.tile_groups + (BOTH ? 0 : my_zero * slot.group_step)) * 16;
        return s;
    }
    // the same of two matrices
    __device__ __forceinline__ TileSource<true> source_of_both(const W4View &v, const uint8_t *m, const W4View &w, const uint8_t *n, int rt, int rt_other, int kt) const {
        TileSource<true> s = source<true>(v, m, rt, kt);
        const TileSource<true> o = source<true>(w, n, rt_other, kt);
        s.other = o.codes;
        if (my_tile == 1) s.scales = o.scales;
        if (my_zero == 1) s.zeros = o.zeros;
        return s;
    }

    // starts the copies of the next slot, which takes one tile or two (BOTH: one of each), and moves the source on
    template <bool BOTH>
    __device__ __forceinline__ void push(TileSource<BOTH> &from, int tiles) {
        const uint32_t s = base + head;
        const bool two = BOTH || tiles == 2;
        copy16(s, from.codes);
        copy16(s + 512, from.codes + 512);
        if (two) {
            const uint8_t *other = BOTH ? from.other : from.codes + W4_TILE_BYTES;
            copy16(s + 1024, other);
            copy16(s + 1536, other + 512);
        }
        const int last = two ? 1 : 0;
        if (my_tile <= last) copy16(s + 2 * W4_TILE_BYTES, from.scales);
        if (my_zero <= last) copy16(s + slot.zeros_at, from.zeros);
        from.codes += tiles * W4_TILE_BYTES;
        if (BOTH) from.other += W4_TILE_BYTES;
        from.scales += tiles * slot.group_step * slot.scale_bytes;
        from.zeros += tiles * slot.group_step * 16;
        close();
    }
    // ends a group of copies (also an empty one, so that groups keep counting slots)
    __device__ __forceinline__ void close() {
        asm volatile("cp.async.commit_group;" ::: "memory");
        head += slot.bytes;
        if (head == end) head = 0;
    }
    // shared address of the oldest slot (this lane's 16 bytes), once it is there (SLOTS - 1 slots are on their way before the call); it
    // may be filled again after the next call
    __device__ __forceinline__ uint32_t pop() {
        asm volatile("cp.async.wait_group %0;" ::"n"(SLOTS - 2) : "memory");
        __syncwarp();
        const uint32_t s = base + tail;
        tail += slot.bytes;
        if (tail == end) tail = 0;
        return s;
    }
};

// shared loads by address; `volatile`: not moved across the ring's waits
__device__ __forceinline__ uint4 lds128(uint32_t a) {
    uint4 v;
    asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(a));
    return v;
}
__device__ __forceinline__ uint2 lds64(uint32_t a) {
    uint2 v;
    asm volatile("ld.shared.v2.u32 {%0, %1}, [%2];" : "=r"(v.x), "=r"(v.y) : "r"(a));
    return v;
}
__device__ __forceinline__ uint32_t lds32(uint32_t a) {
    uint32_t v;
    asm volatile("ld.shared.u32 %0, [%1];" : "=r"(v) : "r"(a));
    return v;
}
__device__ __forceinline__ uint32_t lds16(uint32_t a) {
    uint16_t v;
    asm volatile("ld.shared.u16 %0, [%1];" : "=h"(v) : "r"(a));
    return v;
}

// scales of rows g and g + 8 of the group at `at`
__device__ __forceinline__ float2 slot_scales(uint32_t at, int g, int dtype) {
    if (dtype == MOM_F32) {
        const uint2 b = lds64(at + g * 8);
        return make_float2(__uint_as_float(b.x), __uint_as_float(b.y));
    }
    const uint32_t b = lds32(at + g * 4);
    if (dtype == MOM_BF16) return make_float2(__uint_as_float(b << 16), __uint_as_float(b & 0xffff0000u));
    return __half22float2(*reinterpret_cast<const __half2 *>(&b));
}

// The operand type activations of a type become (bf16 or f16) and the terms an entry enters as: an f32 value is the exact sum of three bf16 values.
template <int DTYPE> struct Operand {
    static constexpr bool BF16 = DTYPE == MOM_F32 || DTYPE == MOM_BF16, EIGHT = DTYPE == MOM_E4M3 || DTYPE == MOM_INT8;
    static constexpr int TERMS = DTYPE == MOM_F32 ? 3 : 1;
};

// The token operand of one tile as a lane sees it: its eight columns of each stretch of 32 (place_of), in
// operand terms.  Rows (this lane's token and columns, at the tile) lie in shared memory or in global memory; term i
// lies i * plane further on.
template <int TERMS>
struct SharedTokens {
    uint32_t row, plane;                       // bytes
    __device__ __forceinline__ uint4 get(int stretch, int term) const { return lds128(row + term * plane + 64 * stretch); }
};
template <int TERMS>
struct GlobalTokens {
    const uint16_t *row;
    long long plane;
    __device__ __forceinline__ uint4 get(int stretch, int term) const {
        return *reinterpret_cast<const uint4 *>(row + term * plane + 32 * stretch);
    }
};
// the same loaded ahead
template <int TERMS>
struct LoadedTokens {
    uint4 b[4][TERMS];
    template <typename TOKENS>
    __device__ __forceinline__ explicit LoadedTokens(const TOKENS &x) {
#pragma unroll
        for (int q = 0; q < 4; ++q)
#pragma unroll
            for (int i = 0; i < TERMS; ++i) b[q][i] = x.get(q, i);
    }
    __device__ __forceinline__ uint4 get(int stretch, int term) const { return b[stretch][term]; }
};

// Scales of 8-bit activations in shared memory: f32 [tokens][stride], from the columns that tile 0 starts with.
struct TokenScales {
    uint32_t at;
    int stride, shift;
};

// Stretches of 32 columns between changes of a scale, at most a tile: 1, 2 or 4.
inline int stretches_per_scale(int group, int x_group) {
    int n = group == 32 || x_group == 32 ? 1 : group == 64 || x_group == 64 ? 2 : 4;
    return n;
}

// sum (accumulator layout of mma.sync: rows g, g + 8 by tokens 2 t, 2 t + 1) += the product of the slot's tile `which` with its token
// operand (kt: the tile's place in the row).
// Every PER stretches of 32 columns the f32 sums of code * x are scaled and added.  EIGHT: 8-bit activations with scales of their own.
template <bool BF16, bool EIGHT, int PER, int TERMS, typename TOKENS>
__device__ __forceinline__ void multiply_tile(const W4View &w, const SlotLayout &l, uint32_t slot, int which, const TOKENS &x, int kt, const TokenScales &xs,
                                              int tokens, float (&sum)[4]) {
    const int lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
    const uint32_t side = which * l.tile_groups;
    const uint4 c[2] = {lds128(slot + which * W4_TILE_BYTES), lds128(slot + which * W4_TILE_BYTES + 512)};
    slot -= lane * 16;
    const int group_stretches = w.group_shift == 5 ? 1 : w.group_shift == 6 ? 2 : 4;
    Offset<BF16> o0, o1;
    o0.set(8);
    o1.set(8);
#pragma unroll
    for (int q0 = 0; q0 < 4; q0 += PER) {
        const int group = PER == 4 ? 0 : q0 / group_stretches;
        if (w.has_zeros) {
            const uint32_t z = lds16(slot + l.zeros_at + (side + group) * 16 + g * 2);
            o0.set(z & 15u);
            o1.set((z >> 8) & 15u);
        }
        const float2 scale = slot_scales(slot + 2 * W4_TILE_BYTES + (side + group) * l.scale_bytes, g, w.scale_dtype);
        // Chains of dependent MMAs: the leading term, and the rest on its own, which would else be cut against sums 2^8 times as large (f32
        // products 1.8e-7 to 2.7e-7 off, apart 0.8e-7); with one term every other stretch.
        constexpr int CHAINS = PER > 1 || TERMS > 1 ? 2 : 1;
        float acc[CHAINS][4];
#pragma unroll
        for (int q = q0; q < q0 + PER; ++q) {
            const uint4 v = c[q >> 1];
            uint32_t a[4], b[4];
            unpack_codes<BF16>(q & 1 ? v.z : v.x, o0, a);
            unpack_codes<BF16>(q & 1 ? v.w : v.y, o1, b);
#pragma unroll
            for (int i = 0; i < TERMS; ++i) {
                const uint4 e = x.get(q, i);
                const int chain = TERMS > 1 ? i > 0 : (q - q0) % CHAINS;
                if (TERMS > 1 ? q == q0 && i < 2 : q - q0 < CHAINS) mma16816_first<BF16>(acc[chain], a[0], b[0], a[1], b[1], e.x, e.y);
                else mma16816<BF16>(acc[chain], a[0], b[0], a[1], b[1], e.x, e.y);
                mma16816<BF16>(acc[chain], a[2], b[2], a[3], b[3], e.z, e.w);
            }
        }
        if (CHAINS == 2)
#pragma unroll
            for (int i = 0; i < 4; ++i) acc[0][i] += acc[CHAINS - 1][i];
        if (EIGHT) {                                       // (sums of tokens that are not there are not used)
            const uint32_t at = xs.at + ((kt * W4_COLS + 32 * q0) >> xs.shift) * 4;
            const float s0 = __uint_as_float(lds32(at + min(2 * t, tokens - 1) * xs.stride * 4));
            const float s1 = __uint_as_float(lds32(at + min(2 * t + 1, tokens - 1) * xs.stride * 4));
            acc[0][0] *= s0; acc[0][1] *= s1; acc[0][2] *= s0; acc[0][3] *= s1;
        }
        sum[0] = fmaf(scale.x, acc[0][0], sum[0]);
        sum[1] = fmaf(scale.x, acc[0][1], sum[1]);
        sum[2] = fmaf(scale.y, acc[0][2], sum[2]);
        sum[3] = fmaf(scale.y, acc[0][3], sum[3]);
    }
}

}  // namespace mom
