// Y = X * W^T (+ T) with W in the 4-bit container on tcgen05, for batches of tokens.
//
// On mma.sync (w4_product.cu) every eight tokens cost as many tensor cycles and shared-memory reads again; here a weight is made into an
// operand once for up to 64 tokens and the rest is the tensor core's.  A CTA takes 128 rows of W (eight row tiles) and N tokens; a
// cluster splits the columns where the row blocks alone do not fill the GPU.  Per step of 128 columns:
//   warps 0-15   two teams that take the steps in turn: codes -> operand entries (exact integers code - zero, w4.cuh) -> TENSOR MEMORY: a container tile already lies in the
//                fragment order of tcgen05.st.16x256b (lane 4 g + t: rows g and g + 8), so that W never passes through
//                shared memory as 16-bit values.  Warp w owns rows 32 (w % 4) .. + 31 (the lanes it may write) and half the columns; its
//                codes come through its own cp.async ring.  (One team alone: 1650 cycles a step, a chain of latencies.)
//   warps 24-27  x -> operand terms -> shared memory, K-major under the 128-byte swizzle: 16-bit rows that are 16-byte addressable by
//                cp.async straight into place, B_STAGES - 1 steps ahead, everything else through registers.
//   warp 28      tcgen05.mma kind::f16 (M128, N, A from tensor memory) into one of two f32 accumulators, a fresh one whenever a
//                scale changes; tcgen05.commit hands out and frees the stages.
//   warps 16-23  the flush: accumulator * scale of the row (* scale of the token) added to f32 sums in registers; at the end the
//                cluster's sums meet in shared memory.
// Measured: 64 tokens, 14336 x 4096 f16 26.4 us (285 TFLOP/s, 1.3 TB/s of W), 36 tokens, 6760 x 9024 in e4m3 54 us, 64 tokens, 8192 x 8192 in
// f32 77 us, 16 tokens, 8192 x 8192 in e4m3 24 us (1.5 TB/s).  29 warps leave 64 registers a thread, and the issue slots that they share bound it,
// with the flush the slowest role (f32 and 8-bit tokens: the staging).  What a role keeps has to be declared inside it: sums of the flush
// that lived through all roles spilled 450 to 1900 bytes a thread (29.3, 104 and 219 us; 4 to 32 bytes are left with 64 tokens, and with 32 in f32).
// Prompts: W is unpacked again for every 64 tokens.  4096 x 4096 in bf16 65 tokens 17.7 us, 128 17.2, 256 23.7, 512 46, 1024 92 us (373 TFLOP/s); in
// e4m3 64 tokens 20 us, 1024 177 us.
// Every wait is bounded; a CTA in which one gives up ends by itself and writes NaN.
#include <algorithm>

#include <cooperative_groups.h>

#include "device_common.cuh"
#include "tc_ptx.cuh"
#include "tc_wait.cuh"
#include "w4_product.h"

namespace mom {

namespace {

namespace cg = cooperative_groups;

constexpr int ROWS = 128, THREADS = 29 * 32, A_STAGES = 4, DEPTH = 8, CODE_DEPTH = 4;
constexpr int UNPACK_WARPS = 16, FLUSH_WARPS = 8, STAGE_WARPS = 4, UNPACK_TEAM = 8;
constexpr int A_COLS = W4_COLS / 2, D_COLS = 64, TMEM_COLS = 512;   // 32-bit columns of a stage of A; of an accumulator (at most)
constexpr int OUT_LD = ROWS + 4;

template <int DTYPE, int N>
struct TcConfig {
    static constexpr int TERMS = Operand<DTYPE>::TERMS;
    static constexpr int B_STAGES = TERMS == 3 ? 2 : 4;
    static constexpr int PANEL = N * 128, B_BYTES = TERMS * 2 * PANEL;       // 64 columns of N tokens; a stage
    static constexpr int CODE_SLOT = 1024 + 64;                              // 64 columns of two row tiles, their zeros
    static constexpr int SIDE_SLOT = 512 + (Operand<DTYPE>::EIGHT ? 4 * N / 2 * 4 : 0);   // scales of two row tiles; of the warp's tokens
    static constexpr int RING_BYTES = UNPACK_WARPS * CODE_DEPTH * CODE_SLOT + FLUSH_WARPS * DEPTH * SIDE_SLOT;
    static constexpr int BARRIERS = 2 * A_STAGES + 2 * B_STAGES + 4;
    static constexpr int SMEM = 1024 + std::max(B_STAGES * B_BYTES, N * OUT_LD * 4) + RING_BYTES + BARRIERS * 8 + 64;
    static_assert(SMEM <= 227 * 1024, "shared memory budget");
    static_assert(2 * D_COLS + A_STAGES * A_COLS <= TMEM_COLS, "tensor memory budget");
};

__device__ __forceinline__ void mma_f16_a_tmem(uint32_t d, uint32_t a, uint64_t b_desc, uint32_t idesc, uint32_t accumulate) {
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}"
        ::"r"(d), "r"(a), "l"(b_desc), "r"(idesc), "r"(accumulate) : "memory");
}
// 16 lanes (rows g and g + 8 of lane 4 g + t) by four blocks of eight columns (2 t, 2 t + 1)
__device__ __forceinline__ void tmem_st_16x256b_x4(uint32_t at, const uint32_t (&r)[16]) {
    asm volatile(
        "tcgen05.st.sync.aligned.16x256b.x4.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16};"
        ::"r"(at), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]), "r"(r[10]),
          "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]) : "memory");
}
// NC consecutive columns of the warp's 32 lanes
template <int NC>
__device__ __forceinline__ void tmem_ld(uint32_t at, float (&v)[NC]) {
    uint32_t r[NC];
    if constexpr (NC == 8)
        asm volatile("tcgen05.ld.sync.aligned.32x32b.x8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                     : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]) : "r"(at) : "memory");
    else
        asm volatile("tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
                     : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]),
                       "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]) : "r"(at) : "memory");
    asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
#pragma unroll
    for (int i = 0; i < NC; ++i) v[i] = __uint_as_float(r[i]);
}
// a += s * x, b += s * y in one instruction
__device__ __forceinline__ void fma_pair(float &a, float &b, float s, float x, float y) {
    asm("{\n\t.reg .b64 p, q, r;\n\tmov.b64 p, {%2, %2};\n\tmov.b64 q, {%3, %4};\n\tmov.b64 r, {%0, %1};\n\tfma.rn.f32x2 r, p, q, r;\n\tmov.b64 {%0, %1}, r;\n\t}"
        : "+f"(a), "+f"(b) : "f"(s), "f"(x), "f"(y));
}
// true in one lane of a converged warp
__device__ __forceinline__ bool elect_one() {
    uint32_t p;
    asm volatile("{\n\t.reg .pred e;\n\telect.sync _|e, 0xffffffff;\n\tselp.u32 %0, 1, 0, e;\n\t}" : "=r"(p));
    return p != 0;
}
__device__ __forceinline__ void copy4(uint32_t dst, const void *src) {
    asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(dst), "l"(src) : "memory");
}
__device__ __forceinline__ void copies_close() { asm volatile("cp.async.commit_group;" ::: "memory"); }
// the oldest of `D` slots has arrived (D - 1 are on their way)
template <int D>
__device__ __forceinline__ void copies_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(D - 2) : "memory"); }

template <int DTYPE, int PER, int N>
__global__ void __launch_bounds__(THREADS, 1) w4_product_tc_kernel(const W4ProductArgs a) {
    using Op = Operand<DTYPE>;
    using C = TcConfig<DTYPE, N>;
    constexpr int FLUSHES = 4 / PER;                           // per step
    extern __shared__ uint8_t raw[];
    uint8_t *smem = reinterpret_cast<uint8_t *>((reinterpret_cast<uintptr_t>(raw) + 1023) & ~(uintptr_t)1023);
    constexpr int FRONT = std::max(C::B_STAGES * C::B_BYTES, N * OUT_LD * 4);
    const uint32_t b_at = ptx::smem_u32(smem), code_at = b_at + FRONT, side_at = code_at + UNPACK_WARPS * CODE_DEPTH * C::CODE_SLOT;
    const uint32_t bars = side_at + FLUSH_WARPS * DEPTH * C::SIDE_SLOT;
    const uint32_t a_full = bars, a_empty = a_full + 8 * A_STAGES, b_full = a_empty + 8 * A_STAGES, b_empty = b_full + 8 * C::B_STAGES,
                   d_full = b_empty + 8 * C::B_STAGES, d_empty = d_full + 16;
    int *words = reinterpret_cast<int *>(smem + FRONT + C::RING_BYTES + C::BARRIERS * 8);   // tensor memory base, abort flag, status (2)
    volatile int *abort_flag = words + 1;
    int32_t *status = words + 2;

    const int warp = __shfl_sync(~0u, threadIdx.x >> 5, 0), lane = threadIdx.x & 31;      // (known to be uniform)
    const W4View &w = a.w;
    const int rank = blockIdx.x % a.split, block = blockIdx.x / a.split, token0 = blockIdx.y * N, tokens = min(N, a.tokens - token0);
    const int ct_first = rank * a.part_tiles, steps = max(0, min(a.part_tiles, w.col_tiles - ct_first));

    if (warp == UNPACK_WARPS + FLUSH_WARPS + STAGE_WARPS) {
        ptx::tmem_alloc(ptx::smem_u32(words), TMEM_COLS);
        ptx::tmem_relinquish();
    }
    if (threadIdx.x == 0) {
        for (int i = 0; i < A_STAGES; ++i) { ptx::mbar_init(a_full + 8 * i, UNPACK_TEAM); ptx::mbar_init(a_empty + 8 * i, 1); }
        for (int i = 0; i < C::B_STAGES; ++i) { ptx::mbar_init(b_full + 8 * i, STAGE_WARPS); ptx::mbar_init(b_empty + 8 * i, 1); }
        for (int i = 0; i < 2; ++i) { ptx::mbar_init(d_full + 8 * i, 1); ptx::mbar_init(d_empty + 8 * i, FLUSH_WARPS); }
        words[1] = words[2] = words[3] = 0;
        ptx::fence_barrier_init();
    }
    ptx::tc_fence_before_sync();
    __syncthreads();
    ptx::tc_fence_after_sync();
    allow_dependents();
    grid_dependency_wait();                                    // nothing has been read from global memory yet
    const uint32_t tmem = __shfl_sync(~0u, (uint32_t)words[0], 0), tmem_a = tmem + 2 * D_COLS;

    constexpr int NC = N / 2;                                  // token columns of a flush warp
    float *out = reinterpret_cast<float *>(smem);              // the sums of 128 rows by N tokens, over the stages of B once they are done with

    if (warp < UNPACK_WARPS) {
        const int quad = warp & 3, half = (warp >> 2) & 1, team = warp / UNPACK_TEAM, g = lane >> 2;
        const uint32_t ring = code_at + warp * CODE_DEPTH * C::CODE_SLOT;
        const int groups = PER == 1 ? 2 : 1, shift = w.group_shift;     // of these 64 columns, as the slot holds them
        const uint8_t *codes[2], *zeros = nullptr;
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int rt = min(block * 8 + quad * 2 + i, w.row_tiles - 1);
            codes[i] = w.base + ((long long)rt * w.col_tiles + ct_first + team) * W4_TILE_BYTES + half * 512 + lane * 16;
        }
        const bool brings = w.has_zeros && lane < 2 * groups;
        if (brings) zeros = w.base + w.zeros_at + (long long)min(block * 8 + quad * 2 + lane / groups, w.row_tiles - 1) * w.groups * 16;
        uint32_t fill = ring + lane * 16, use = ring;
        auto fetch = [&](int step) {
            if (step < steps) {
                const uint32_t s = fill - lane * 16;
                copy16(fill, codes[0]);
                copy16(fill + 512, codes[1]);
                codes[0] += 2 * W4_TILE_BYTES;
                codes[1] += 2 * W4_TILE_BYTES;
                fill += C::CODE_SLOT;
                if (fill == ring + lane * 16 + CODE_DEPTH * C::CODE_SLOT) fill = ring + lane * 16;
                if (brings) {
                    const int k = (ct_first + step) * W4_COLS + half * 64 + (lane % groups) * 32;
                    copy16(s + 1024 + lane * 16, zeros + (long long)min(k >> shift, w.groups - 1) * 16);
                }
            }
            copies_close();
        };
        for (int i = 0; i < CODE_DEPTH - 1; ++i) fetch(team + 2 * i);
        for (int step = team; step < steps; step += 2) {
            copies_wait<CODE_DEPTH>();
            __syncwarp();
            const uint32_t s = use;
            use += C::CODE_SLOT;
            if (use == ring + CODE_DEPTH * C::CODE_SLOT) use = ring;
            const int stage = step % A_STAGES;
            uint32_t r[2][16];
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const uint4 c = lds128(s + i * 512 + lane * 16);
                Offset<Op::BF16> o0, o1;
                o0.set(8);
                o1.set(8);
#pragma unroll
                for (int q = 0; q < 2; ++q) {
                    if (w.has_zeros && (q == 0 || PER == 1)) {
                        const uint32_t z = lds16(s + 1024 + (i * groups + q) * 16 + g * 2);
                        o0.set(z & 15u);
                        o1.set((z >> 8) & 15u);
                    }
                    uint32_t p[4], v[4];
                    unpack_codes<Op::BF16>(q ? c.z : c.x, o0, p);
                    unpack_codes<Op::BF16>(q ? c.w : c.y, o1, v);
#pragma unroll
                    for (int b = 0; b < 2; ++b) {
                        r[i][8 * q + 4 * b] = p[2 * b];
                        r[i][8 * q + 4 * b + 1] = p[2 * b + 1];
                        r[i][8 * q + 4 * b + 2] = v[2 * b];
                        r[i][8 * q + 4 * b + 3] = v[2 * b + 1];
                    }
                }
            }
            if (step >= A_STAGES && !wait_barrier(a_empty + 8 * stage, (step / A_STAGES - 1) & 1, abort_flag, status, 1)) break;
            ptx::tc_fence_after_sync();
#pragma unroll
            for (int i = 0; i < 2; ++i)
                tmem_st_16x256b_x4(tmem_a + ((uint32_t)(quad * 32 + i * 16) << 16) + stage * A_COLS + half * 32, r[i]);
            ptx::tmem_wait_st();
            ptx::tc_fence_before_sync();
            __syncwarp();
            if (lane == 0) ptx::mbar_arrive(a_full + 8 * stage);
            fetch(step + 2 * (CODE_DEPTH - 1));
        }
    } else if (warp < UNPACK_WARPS + FLUSH_WARPS) {
        const int quad = warp & 3, part = (warp - UNPACK_WARPS) >> 2, scale_bytes = w.scale_dtype == MOM_F32 ? 64 : 32;
        const uint32_t ring = side_at + (warp - UNPACK_WARPS) * DEPTH * C::SIDE_SLOT;
        const int groups = w.group_shift >= 7 ? 1 : W4_COLS >> w.group_shift;                // of a step, as the slot holds them
        const int x_groups = a.x_group_shift >= 7 ? 1 : W4_COLS >> a.x_group_shift;
        const int per = scale_bytes / 16, pieces = 2 * groups * per;
        const uint8_t *scales = w.base + w.scales_at + (long long)min(block * 8 + quad * 2 + lane / (groups * per), w.row_tiles - 1) * w.groups * scale_bytes + lane % per * 16;
        const int my_group = lane / per % groups;
        const float *token_scales = Op::EIGHT ? a.x_scales + (long long)(token0 + min(part * NC + lane % NC, tokens - 1)) * a.x_groups : nullptr;
        auto fetch = [&](int step) {
            if (step < steps) {
                const uint32_t s = ring + (step % DEPTH) * C::SIDE_SLOT;
                const int k = (ct_first + step) * W4_COLS;
                if (lane < pieces) copy16(s + lane * 16, scales + (long long)min((k >> w.group_shift) + my_group, w.groups - 1) * scale_bytes);
                if (Op::EIGHT && lane < NC)
                    for (int i = 0; i < x_groups; ++i)
                        copy4(s + 512 + (i * NC + lane) * 4, token_scales + min((k >> a.x_group_shift) + i, a.x_groups - 1));
            }
            copies_close();
        };
        for (int i = 0; i < DEPTH - 1; ++i) fetch(i);
        const int r = lane & 15, at = ((r & 7) * 2 + (r >> 3));
        float sum[NC] = {};                                    // (declared here: the other roles need the registers)
        bool fine = true;
        for (int step = 0; step < steps && fine; ++step) {
            copies_wait<DEPTH>();
            __syncwarp();
            const uint32_t s = ring + (step % DEPTH) * C::SIDE_SLOT;
#pragma unroll
            for (int f = 0; f < FLUSHES; ++f) {
                const int n = step * FLUSHES + f, d = n & 1;
                const int group = f * PER * groups / 4;
                const uint32_t entry = s + ((lane >> 4) * groups + group) * scale_bytes;
                float scale;
                if (w.scale_dtype == MOM_F32) scale = __uint_as_float(lds32(entry + at * 4));
                else if (w.scale_dtype == MOM_BF16) scale = __uint_as_float(lds16(entry + at * 2) << 16);
                else scale = __half2float(__ushort_as_half((unsigned short)lds16(entry + at * 2)));
                if (!wait_barrier(d_full + 8 * d, (n >> 1) & 1, abort_flag, status, 2)) { fine = false; break; }
                ptx::tc_fence_after_sync();
                constexpr int AT_ONCE = NC == 16 ? 16 : 8;                                   // (registers)
#pragma unroll
                for (int c = 0; c < NC; c += AT_ONCE) {
                    float v[AT_ONCE];
                    tmem_ld<AT_ONCE>(tmem + ((uint32_t)(quad * 32) << 16) + d * D_COLS + part * NC + c, v);
                    if (c + AT_ONCE == NC) {
                        ptx::tc_fence_before_sync();
                        __syncwarp();
                        if (lane == 0) ptx::mbar_arrive(d_empty + 8 * d);
                    }
                    if (Op::EIGHT) {
                        const uint32_t t = s + 512 + ((f * PER * x_groups / 4) * NC + c) * 4;
#pragma unroll
                        for (int i = 0; i < AT_ONCE; i += 4) {
                            const uint4 b = lds128(t + i * 4);
                            v[i] *= __uint_as_float(b.x); v[i + 1] *= __uint_as_float(b.y);
                            v[i + 2] *= __uint_as_float(b.z); v[i + 3] *= __uint_as_float(b.w);
                        }
                    }
#pragma unroll
                    for (int i = 0; i < AT_ONCE; i += 2) fma_pair(sum[c + i], sum[c + i + 1], scale, v[i], v[i + 1]);
                }
            }
            fetch(step + DEPTH - 1);
        }
        // the last accumulator has been flushed, so that every MMA has read its operands and all staging is over
        if (fine)
#pragma unroll
            for (int i = 0; i < NC; ++i) out[(part * NC + i) * OUT_LD + quad * 32 + lane] = sum[i];
    } else if (warp < UNPACK_WARPS + FLUSH_WARPS + STAGE_WARPS) {
        // eight entries at a time: token thread / 16 + 8 j, columns 8 (thread % 16) .. + 7 of the step
        constexpr int PIECES = N * (W4_COLS / 8) / (STAGE_WARPS * 32);
        const int thread = threadIdx.x - (UNPACK_WARPS + FLUSH_WARPS) * 32, token = thread >> 4, piece = thread & 15;
        const uint32_t to = b_at + (piece >> 3) * C::PANEL + token * 128 + (((piece & 7) ^ (token & 7)) << 4);      // (tokens 8 j on: 1024 j bytes on)
        const typename Element<DTYPE>::type *x = static_cast<const typename Element<DTYPE>::type *>(a.x);
        // (addresses are made where they are used: an array of them does not fit into the registers of 64 tokens; the tokens that are not there read the last one)
        const typename Element<DTYPE>::type *first = x + (long long)(token0 + token) * a.x_stride;
        const int last = tokens - 1 - token;
        auto row = [&](int j) { return first + min(8 * j, last) * a.x_stride; };
        if (sizeof(*x) == 2 && a.wide && w.cols % 8 == 0) {
            auto fetch = [&](int step) {
                if (step < steps) {
                    // (columns beyond the last: 0 of 16 bytes are read, the rest is filled with zeros)
                    const int k = (ct_first + step) * W4_COLS + piece * 8, bytes = k < w.cols ? 16 : 0, at = bytes ? k : 0;
                    const uint32_t s = to + step % C::B_STAGES * C::B_BYTES;
#pragma unroll
                    for (int j = 0; j < PIECES; ++j)
                        asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(s + 1024 * j), "l"(row(j) + at), "r"(bytes) : "memory");
                }
                copies_close();
            };
            for (int i = 0; i < C::B_STAGES - 1; ++i) fetch(i);
            for (int step = 0; step < steps; ++step) {
                asm volatile("cp.async.wait_group %0;" ::"n"(C::B_STAGES - 2) : "memory");
                ptx::fence_proxy_async_smem();
                __syncwarp();
                if (lane == 0) ptx::mbar_arrive(b_full + 8 * (step % C::B_STAGES));
                // the stage of the step before is filled next, once its MMAs are done
                if (step > 0 && step + C::B_STAGES - 1 < steps &&
                    !wait_barrier(b_empty + 8 * ((step - 1) % C::B_STAGES), ((step - 1) / C::B_STAGES) & 1, abort_flag, status, 3))
                    break;
                fetch(step + C::B_STAGES - 1);
            }
        } else {
            // HOLD pieces at a time, two such batches on their way (32 registers)
            constexpr int WORDS = sizeof(Raw8<DTYPE>) / 4, HOLD = std::min(PIECES, 16 / WORDS), BATCHES = PIECES / HOLD, TURN = std::max(2, BATCHES);
            static_assert(PIECES % HOLD == 0 && TURN % 2 == 0 && TURN % BATCHES == 0, "batches of a step, in turn");
            Raw8<DTYPE> held[2][HOLD];
            auto load = [&](int batch, Raw8<DTYPE> (&v)[HOLD]) {               // (beyond the last column: zeros, nothing is read)
                const int k = (ct_first + batch / BATCHES) * W4_COLS + piece * 8, j0 = batch % BATCHES * HOLD;
#pragma unroll
                for (int j = 0; j < HOLD; ++j) v[j] = load_x8<DTYPE>(row(j0 + j), k, w.cols, a.wide);
            };
            load(0, held[0]);
            load(1, held[1]);
            bool fine = true;
            for (int batch0 = 0; batch0 < steps * BATCHES && fine; batch0 += TURN) {
#pragma unroll
                for (int i = 0; i < TURN; ++i) {
                    const int step = (batch0 + i) / BATCHES, stage = step % C::B_STAGES;
                    if (step >= steps) break;
                    if (i % BATCHES == 0 && step >= C::B_STAGES &&
                        !(fine = wait_barrier(b_empty + 8 * stage, (step / C::B_STAGES - 1) & 1, abort_flag, status, 3)))
                        break;
                    const uint32_t s = to + stage * C::B_BYTES + i % BATCHES * HOLD * 1024;
#pragma unroll
                    for (int j = 0; j < HOLD; ++j) {
                        uint32_t b[Op::TERMS][4];
                        expand_x8<DTYPE, Op::TERMS>(held[i & 1][j], b);
#pragma unroll
                        for (int q = 0; q < Op::TERMS; ++q)
                            asm volatile("st.shared.v4.u32 [%0], {%1, %2, %3, %4};" ::"r"(s + q * 2 * C::PANEL + 1024 * j), "r"(b[q][0]), "r"(b[q][1]),
                                         "r"(b[q][2]), "r"(b[q][3]) : "memory");
                    }
                    load(batch0 + i + 2, held[i & 1]);
                    if (i % BATCHES == BATCHES - 1) {
                        ptx::fence_proxy_async_smem();
                        __syncwarp();
                        if (lane == 0) ptx::mbar_arrive(b_full + 8 * stage);
                    }
                }
            }
        }
    } else {
        // the whole warp walks the loop, so that addresses and descriptors stay in uniform registers; one elected lane issues
        constexpr uint32_t type = Op::BF16 ? 1u : 0u;
        constexpr uint32_t idesc = (1u << 4) | (type << 7) | (type << 10) | ((uint32_t)(N >> 3) << 17) | ((uint32_t)(ROWS >> 4) << 24);
        const uint64_t desc0 = ptx::smem_desc(b_at, 16, 1024, ptx::SWIZZLE_128B);      // + (bytes further on) / 16
        bool fine = true;
        for (int step = 0; step < steps && fine; ++step) {
            const int sa = step % A_STAGES, sb = step % C::B_STAGES;
            const uint64_t desc = desc0 + (uint32_t)(sb * (C::B_BYTES / 16));
            const uint32_t a_at = tmem_a + sa * A_COLS;
            fine = wait_barrier(a_full + 8 * sa, (step / A_STAGES) & 1, abort_flag, status, 4) &&
                   wait_barrier(b_full + 8 * sb, (step / C::B_STAGES) & 1, abort_flag, status, 5);
#pragma unroll
            for (int f = 0; f < FLUSHES; ++f) {
                const int n = step * FLUSHES + f, d = n & 1;
                if (!fine) break;
                if (n >= 2 && !(fine = wait_barrier(d_empty + 8 * d, ((n >> 1) - 1) & 1, abort_flag, status, 6))) break;
                ptx::tc_fence_after_sync();
                if (elect_one()) {
                    // (f32 tokens: the small terms of all columns first, so that their sums are not cut against those of the leading one)
#pragma unroll
                    for (int t = Op::TERMS - 1; t >= 0; --t)
#pragma unroll
                        for (int q = 0; q < 2 * PER; ++q) {    // 16 columns each
                            const int k = f * 2 * PER + q;
                            mma_f16_a_tmem(tmem + d * D_COLS, a_at + k * 8, desc + ((t * 2 + (k >> 2)) * C::PANEL + (k & 3) * 32) / 16, idesc,
                                           q > 0 || t < Op::TERMS - 1);
                        }
                    ptx::mma_commit(d_full + 8 * d);
                    if (f == FLUSHES - 1) {
                        ptx::mma_commit(a_empty + 8 * sa);
                        ptx::mma_commit(b_empty + 8 * sb);
                    }
                }
                __syncwarp();
            }
        }
    }
    asm volatile("cp.async.wait_all;" ::: "memory");
    __syncwarp();
    ptx::tc_fence_before_sync();
    __syncthreads();
    ptx::tc_fence_after_sync();

    // the CTA's sums, then the cluster's in the order of its CTAs
    if (*abort_flag)
        for (int i = threadIdx.x; i < N * OUT_LD; i += THREADS) out[i] = __int_as_float(0x7fffffff);
    if (warp == UNPACK_WARPS + FLUSH_WARPS + STAGE_WARPS) ptx::tmem_dealloc(tmem, TMEM_COLS);
    if (a.split > 1) ptx::cluster_sync();
    else __syncthreads();
    // a thread finishes four tokens of a row at a time, the loads of T and of the cluster's sums all under way before the first is used
    const int per_rank = ROWS / a.split, r = threadIdx.x % per_rank, row = rank * per_rank + r, n = block * ROWS + row;
    const int lanes = THREADS / per_rank, first = threadIdx.x / per_rank;
    if (first < lanes && n < w.rows) {
        for (int t0 = first; t0 < tokens; t0 += 4 * lanes) {
            float v[4], add[4] = {0.0f, 0.0f, 0.0f, 0.0f};
            if (a.add) load_batch(a.add, a.y_dtype, [&](int j) { return (token0 + min(t0 + j * lanes, tokens - 1)) * a.add_stride + n; }, add);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int token = min(t0 + j * lanes, tokens - 1);
                v[j] = 0.0f;
                if (a.split == 1) v[j] = out[token * OUT_LD + row];
                else
                    for (int p = 0; p < a.split; ++p) v[j] += *cg::this_cluster().map_shared_rank(out + token * OUT_LD + row, p);
            }
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int token = t0 + j * lanes;
                if (token < tokens) store_from_float(a.y, (token0 + token) * a.y_stride + n, a.y_dtype, v[j] + add[j]);
            }
        }
    }
    if (a.split > 1) ptx::cluster_sync();
}

template <int DTYPE, int PER, int N>
cudaError_t launch(W4ProductArgs a, int sm_count, cudaStream_t stream) {
    using C = TcConfig<DTYPE, N>;
    cudaError_t e = raise_smem_limit<w4_product_tc_kernel<DTYPE, PER, N>>(C::SMEM);
    if (e != cudaSuccess) return e;
    const int blocks = (a.w.row_tiles + 7) / 8, token_blocks = (a.tokens + N - 1) / N;
    // Columns split over a cluster where that shortens the launch: waves of clusters times steps, each CTA paying START steps to begin and end.
    constexpr int START = 12;
    long long best = 0;
    a.split = 1;
    for (int split = 1; split <= 8; split *= 2) {
        const int room = split == 1 ? sm_count : resident_clusters<w4_product_tc_kernel<DTYPE, PER, N>>(split, THREADS, C::SMEM);
        if (room < 1 || (split > 1 && a.w.col_tiles < 2 * split)) continue;
        const long long waves = ((long long)blocks * token_blocks + room - 1) / room, cost = waves * ((a.w.col_tiles + split - 1) / split + START);
        if (split == 1 || cost < best) { best = cost; a.split = split; }
    }
    a.part_tiles = (a.w.col_tiles + a.split - 1) / a.split;
    return launch_dependent(w4_product_tc_kernel<DTYPE, PER, N>, dim3(blocks * a.split, token_blocks), dim3(THREADS), C::SMEM, stream, a.split, a);
}

template <int DTYPE, int PER>
cudaError_t launch(const W4ProductArgs &a, int sm_count, cudaStream_t stream) {
    return a.tokens <= 16 ? launch<DTYPE, PER, 16>(a, sm_count, stream) : a.tokens <= 32 ? launch<DTYPE, PER, 32>(a, sm_count, stream)
                                                                                           : launch<DTYPE, PER, 64>(a, sm_count, stream);
}

template <int DTYPE>
cudaError_t launch(const W4ProductArgs &a, int per, int sm_count, cudaStream_t stream) {
    return per == 1 ? launch<DTYPE, 1>(a, sm_count, stream) : per == 2 ? launch<DTYPE, 2>(a, sm_count, stream) : launch<DTYPE, 4>(a, sm_count, stream);
}

}  // namespace

cudaError_t launch_w4_product_tc(const W4ProductArgs &a, int x_dtype, int per, int sm_count, cudaStream_t stream) {
    switch (x_dtype) {
        case MOM_F32: return launch<MOM_F32>(a, per, sm_count, stream);
        case MOM_BF16: return launch<MOM_BF16>(a, per, sm_count, stream);
        case MOM_F16: return launch<MOM_F16>(a, per, sm_count, stream);
        case MOM_E4M3: return launch<MOM_E4M3>(a, per, sm_count, stream);
        default: return launch<MOM_INT8>(a, per, sm_count, stream);
    }
}

}  // namespace mom
