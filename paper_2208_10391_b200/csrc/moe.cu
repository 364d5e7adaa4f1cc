// A mixture-of-experts layer for a few tokens in one launch (formulas in include/mom.h).
//
// One CTA per SM, all resident (cooperative launch), three stages with a barrier over the grid between them:
//   1  the router's products; the logits go to the workspace.  16-bit x and R run on mma.sync (16 experts by 8 tokens, the warps share the
//      columns), anything else on FFMA (four warps share an expert's row for eight tokens).
//   2  every CTA ranks every token's experts for itself (a warp per token: softmax in registers, top_k rounds of one
//      warp-wide reduction and a ballot; cheaper than a further barrier).  Then each CTA takes a run of the (8 tokens of an expert, 16 rows of
//      G and of U) units; the tokens are staged in shared memory as operand terms, once for all of the run's rows; its warps
//      take even stretches of the rows' tiles (w4.cuh), rows that two or more share are put together from their parts, and
//      h = silu(G x) * (U x) goes to the workspace as operand planes, three bf16 terms that hold all of it.
//   3  the CTAs deal out the 16-row tiles of D (two at a time where there are enough, so that h is read half as often): the
//      warps take even stretches of all chosen experts' tiles, D h lands in shared memory by (token, expert), and y adds
//      share * D h over a token's experts in their order: no atomics, the same bits every time.  The first tiles of D are
//      on their way before the barrier is waited for.  Where D has fewer rows than the GPU has SMs, several CTAs share a row's tiles
//      and their parts of y are added after a further barrier.
// Measured: 64 tokens, 64 experts of 4096 x 1280 251 us (520 MB: 2.1 TB/s; the 92 blocks of eight tokens that the experts get are each a pass
// over the instructions of w4.cuh, which bound it), in f32 411 us; one token, 64 experts of 2048 x 1024, 25.5 us, a chain of latencies: router 4K
// cycles, ranking 4K, G and U 15K, D 8K and two barriers; 5 tokens, 10 experts of 1001 x 333 in f32 23.5 us; 45 tokens, 83 experts of 320 x 558
// in f32 48 us.
// Only the chosen experts' weights are read.  Every wait is bounded; a CTA that gives up records it and still arrives at the next barrier, so
// that nobody waits for it; it writes NaN for its part of y, and so do all that meet it at a later barrier.
#include <algorithm>
#include <cmath>

#include <mutex>
#include <new>

#include "tc_wait.cuh"
#include "w4.cuh"

struct mom_moe_plan {
    mom_moe_desc_t desc;
    mom_w4_desc_t gate, down;                // U has G's
    mutable std::mutex mutex;
    mutable int device = -1;
    mutable unsigned long long *block = nullptr;   // [0] barrier arrivals, then the status words
    mutable unsigned long long probe_ns = 0;       // self-test: the next execute's waits run out after so long
};

namespace mom {

namespace {

constexpr int WARPS = 16, THREADS = 32 * WARPS, SLOTS = 3;
constexpr int MAX_T = MOM_MOE_MAX_TOKENS, MAX_E = MOM_MOE_MAX_EXPERTS, MAX_K = MOM_MOE_MAX_TOP_K, MAX_PAIRS = MOM_MOE_MAX_PAIRS;
constexpr int MAX_WIDTH = MOM_MOE_MAX_WIDTH;     // keeps a CTA's tiles, times its warps, in 32 bits
constexpr int LD = W4_ROWS + 1, TOKENS = 8;      // of a unit: one token operand of mma.sync
constexpr int BATCH = 16;                        // rows of a run whose sums over chunks of columns are kept at a time
constexpr int SHARED_LIMIT = 227 * 1024;
constexpr int MAX_SPLITS = 8;                    // CTAs that share the tiles of a row of D

struct MoeArgs {
    W4View gate, up, down;
    const void *x, *router;
    void *y;
    long long x_stride, y_stride;
    int tokens, hidden, inner, experts, top_k, renormalize, dtype, router_dtype, wide;
    int h_cols;                    // row length of the planes of h, whole tiles
    int resident, chunk_tiles;     // x of all tokens is staged once; column tiles of x staged at a time
    int pair_rows;                 // stage 3 takes two row tiles at a time
    float *logits;                 // workspace: [tokens][experts]
    uint16_t *h_planes;            // [terms][tokens * top_k][h_cols], in the order of place_of
    float *parts;                  // [MAX_SPLITS][tokens][hidden]
    int32_t *ids;
    float *shares;
    unsigned long long *arrivals;
    int32_t *status;
    unsigned long long limit_ns;
    int missing;                   // self-test: arrivals that are waited for and never come
};

constexpr int H_TERMS = 3;                       // of h as the operand of D (bf16): all 24 bits in layers of every type (64 tokens with two terms, 2^-18 off, 229 us, with three 251)

// Up to eight tokens of one expert.
struct Block {
    short expert, first_row, rows;             // rows of h: (token, expert) pairs in the order of experts, then tokens
};
struct alignas(16) Routing {
    unsigned long long chosen[MAX_E];          // bit t: token t chose the expert
    short first[MAX_E];                        // the expert's first row of h
    Block blocks[MAX_PAIRS];
    unsigned char token[MAX_PAIRS];            // of a row of h
    short ids[MAX_T][MAX_K], row[MAX_T][MAX_K];    // a token's experts, its rows of h
    float shares[MAX_T][MAX_K];
    int n_blocks, fine;                        // fine: no wait of this launch is known to have given up
};
// Shared memory: Routing, the warps' rings, then by stage
//   1  Slots                                             2  Part, sums over chunks (where x is staged in chunks), x
//   3  D h by row of h [1 or 2 row tiles][rows][LD], DownPart
// x that is staged before stage 2 (resident) lies behind Part.
union Slots {
    float mma[WARPS][W4_ROWS][TOKENS + 1], fma[4][4][TOKENS];
};
struct Part { float v[WARPS][2][2][TOKENS][LD]; };              // a stretch's first and last row; G, U
struct Sums { float v[BATCH][2][TOKENS][LD]; };
template <int ROWS> struct DownPart { float v[WARPS][2][ROWS][TOKENS][LD]; };

// All CTAs of the grid meet.  The count (the lower 48 bits) only grows and every CTA of every launch arrives at every barrier, so that it is a
// multiple of the grid between launches: targets count on from the multiple that was read when the kernel began.  A CTA whose wait gave
// up adds to the upper bits with all its later arrivals, so that everyone who meets it there learns of it without a further load.
constexpr unsigned long long GAVE_UP = 1ull << 48, COUNT = GAVE_UP - 1;
__device__ __forceinline__ void grid_arrive(const MoeArgs &a, const Routing &r) {
    __syncthreads();
    if (threadIdx.x == 0)
        asm volatile("fence.acq_rel.gpu;\n\tred.relaxed.gpu.global.add.u64 [%0], %1;" ::"l"(a.arrivals), "l"(r.fine ? 1ull : GAVE_UP + 1) : "memory");
}
// `begun`: what the count was when the launch began.  Clears r.fine once a wait of the launch has given up: one of this CTA, or of another
// before it arrived here.
__device__ __forceinline__ void grid_wait(const MoeArgs &a, Routing &r, unsigned long long begun, int barrier) {
    if (threadIdx.x == 0) {
        const unsigned long long target = (begun & COUNT) + (unsigned)barrier * gridDim.x + a.missing;
        unsigned long long start = 0, seen;
        for (unsigned i = 0;; ++i) {
            asm volatile("ld.acquire.gpu.global.u64 %0, [%1];" : "=l"(seen) : "l"(a.arrivals) : "memory");
            if ((seen & COUNT) >= target) break;
            if ((i & 63) == 63) {
                const unsigned long long now = global_ns();
                if (start == 0) start = now;
                else if (now - start > a.limit_ns) {
                    if (atomicCAS(a.status, 0, (int)MOM_ERR_DEVICE_TIMEOUT) == 0) a.status[1] = barrier;
                    r.fine = 0;
                    break;
                }
            }
        }
        if ((seen ^ begun) >= GAVE_UP) r.fine = 0;
    }
    __syncthreads();
}

// v as three bf16 terms, which hold all of it
__device__ __forceinline__ void store_terms(uint16_t *p, long long plane, float v) {
    uint32_t t0, t1, t2;
    split_pair(v, 0.0f, t0, t1, t2);
    p[0] = (uint16_t)t0; p[plane] = (uint16_t)t1; p[2 * plane] = (uint16_t)t2;
}

// ---- stage 1
template <int DTYPE>
__device__ void route_mma(const MoeArgs &a, Slots &slots) {
    using T = typename Element<DTYPE>::type;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, g = lane >> 2, t = lane & 3;
    const int chunks = (a.tokens + 7) / 8, items = (a.experts + 15) / 16 * chunks, stretches = (a.hidden + 31) / 32;
    const bool r_wide = aligned_16(a.router) && a.hidden % 8 == 0;
    for (int item = blockIdx.x; item < items; item += gridDim.x) {
        const int e0 = item / chunks * 16, t0 = (item - e0 / 16 * chunks) * 8;
        const T *r0 = static_cast<const T *>(a.router) + (long long)min(e0 + g, a.experts - 1) * a.hidden;      // (what is not there: computed, not used)
        const T *r1 = static_cast<const T *>(a.router) + (long long)min(e0 + g + 8, a.experts - 1) * a.hidden;
        const T *x = static_cast<const T *>(a.x) + min(t0 + g, a.tokens - 1) * a.x_stride;
        float c[2][4] = {};
        for (int s0 = warp; s0 < stretches; s0 += 4 * WARPS) {
            Raw8<DTYPE> p[4], q[4], v[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int k = (s0 + j * WARPS) * 32 + 8 * t;              // (beyond the last column: zeros, nothing is read)
                p[j] = load_x8<DTYPE>(r0, k, a.hidden, r_wide);
                q[j] = load_x8<DTYPE>(r1, k, a.hidden, r_wide);
                v[j] = load_x8<DTYPE>(x, k, a.hidden, a.wide);
            }
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                mma16816<DTYPE == MOM_BF16>(c[0], p[j].r[0], q[j].r[0], p[j].r[1], q[j].r[1], v[j].r[0], v[j].r[1]);
                mma16816<DTYPE == MOM_BF16>(c[1], p[j].r[2], q[j].r[2], p[j].r[3], q[j].r[3], v[j].r[2], v[j].r[3]);
            }
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) slots.mma[warp][g + 8 * (i >> 1)][2 * t + (i & 1)] = c[0][i] + c[1][i];
        __syncthreads();
        if (threadIdx.x < 128) {
            const int e = threadIdx.x >> 3, token = threadIdx.x & 7;
            float v = 0.0f;
#pragma unroll
            for (int w = 0; w < WARPS; ++w) v += slots.mma[w][e][token];
            if (e0 + e < a.experts && t0 + token < a.tokens) a.logits[(t0 + token) * a.experts + e0 + e] = v;
        }
        __syncthreads();
    }
}

template <typename T, typename R>
__device__ void route_fma(const MoeArgs &a, Slots &slots) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, team = warp >> 2, part = warp & 3;
    const int chunks = (a.tokens + 7) / 8, items = a.experts * chunks;
    for (int i0 = blockIdx.x * 4; i0 < items; i0 += gridDim.x * 4) {
        const int item = min(i0 + team, items - 1), e = item / chunks, t0 = (item - e * chunks) * 8;
        const R *r = static_cast<const R *>(a.router) + (long long)e * a.hidden;
        const T *x = static_cast<const T *>(a.x);
        float s[8] = {};
        for (int k0 = part * 32 + lane; k0 < a.hidden; k0 += 512) {       // four columns at a time, all loads under way before the first is used
            R rv[4];
            T xv[4][8];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int k = min(k0 + 128 * i, a.hidden - 1);
                rv[i] = r[k];
#pragma unroll
                for (int j = 0; j < 8; ++j) xv[i][j] = x[min(t0 + j, a.tokens - 1) * a.x_stride + k];
            }
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (k0 + 128 * i < a.hidden)
#pragma unroll
                    for (int j = 0; j < 8; ++j) s[j] = fmaf(to_float(rv[i]), to_float(xv[i][j]), s[j]);
        }
#pragma unroll
        for (int j = 0; j < 8; ++j)
#pragma unroll
            for (int o = 16; o; o >>= 1) s[j] += __shfl_xor_sync(~0u, s[j], o);
        if (lane == 0)
#pragma unroll
            for (int j = 0; j < 8; ++j) slots.fma[team][part][j] = s[j];
        __syncthreads();
        if (threadIdx.x < 32) {
            const int q = threadIdx.x >> 3, j = threadIdx.x & 7, it = i0 + q;
            if (it < items) {
                const int ee = it / chunks, token = (it - ee * chunks) * 8 + j;
                if (token < a.tokens) a.logits[token * a.experts + ee] = (slots.fma[q][0][j] + slots.fma[q][1][j]) + (slots.fma[q][2][j] + slots.fma[q][3][j]);
            }
        }
        __syncthreads();
    }
}

// the columns of h's planes that no unit writes
__device__ void fill_planes(const MoeArgs &a) {
    const int written = a.gate.row_tiles * W4_ROWS, rest = a.h_cols - written;
    const int rows = H_TERMS * a.tokens * a.top_k;
    for (int row = blockIdx.x; row < rows; row += gridDim.x)
        for (int i = threadIdx.x; i < rest; i += THREADS) a.h_planes[(long long)row * a.h_cols + place_of(written + i)] = 0;
}

// ---- stage 2: which experts
// order-preserving map of the probabilities (0 .. 1) to integers above 1; NaN: 1
__device__ __forceinline__ uint32_t rank_key(float p) { return p >= 0.0f ? __float_as_uint(p) + 2u : 1u; }
__device__ __forceinline__ float rank_value(uint32_t key) { return key >= 2u ? __uint_as_float(key - 2u) : __int_as_float(0x7fffffff); }

// softmax and top_k of every token, J = ceil(experts / 32) values a lane
template <int J>
__device__ void rank_tokens(const MoeArgs &a, Routing &r) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    for (int t = warp; t < a.tokens; t += WARPS) {
        float p[J];
        float top = -INFINITY;
#pragma unroll
        for (int j = 0; j < J; ++j) {
            const int e = lane + 32 * j;
            p[j] = e < a.experts ? __ldcg(a.logits + t * a.experts + e) : -INFINITY;
        }
#pragma unroll
        for (int j = 0; j < J; ++j) top = max_nan(top, p[j]);
#pragma unroll
        for (int o = 16; o; o >>= 1) top = max_nan(top, __shfl_xor_sync(~0u, top, o));
        float sum = 0.0f;
#pragma unroll
        for (int j = 0; j < J; ++j) {
            p[j] = lane + 32 * j < a.experts ? expf(p[j] - top) : 0.0f;
            sum += p[j];
        }
#pragma unroll
        for (int o = 16; o; o >>= 1) sum += __shfl_xor_sync(~0u, sum, o);
        uint32_t key[J];                                       // 0: taken, or no expert; NaN ranks below every number
#pragma unroll
        for (int j = 0; j < J; ++j) key[j] = lane + 32 * j < a.experts ? rank_key(p[j] / sum) : 0u;
        float mine = 0.0f, total = 0.0f;                       // lane i keeps the i-th share
        int mine_id = 0;
        for (int i = 0; i < a.top_k; ++i) {
            uint32_t best = key[0];
            int at = lane;
#pragma unroll
            for (int j = 1; j < J; ++j)
                if (key[j] > best) { best = key[j]; at = lane + 32 * j; }
            const uint32_t most = __reduce_max_sync(~0u, best);
            const unsigned have = __ballot_sync(~0u, best == most);
            int e = __shfl_sync(~0u, at, __ffs(have) - 1);
            if (J > 1 && (have & (have - 1))) e = (int)__reduce_min_sync(~0u, best == most ? (unsigned)at : 0x7fffffffu);
#pragma unroll
            for (int j = 0; j < J; ++j)
                if (lane + 32 * j == e) key[j] = 0;
            const float share = rank_value(most);
            total += share;
            if (lane == i) { mine = share; mine_id = e; }
        }
        if (lane < a.top_k) {
            atomicOr(&r.chosen[mine_id], 1ull << t);
            if (a.renormalize) mine /= total;
            r.ids[t][lane] = (short)mine_id;
            r.shares[t][lane] = mine;
            if (blockIdx.x == 0) {
                if (a.ids) a.ids[t * a.top_k + lane] = mine_id;
                if (a.shares) a.shares[t * a.top_k + lane] = mine;
            }
        }
    }
}

// (r.chosen is cleared before the barrier)
__device__ void rank_experts(const MoeArgs &a, Routing &r) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    if (a.experts <= 32) rank_tokens<1>(a, r);
    else if (a.experts <= 64) rank_tokens<2>(a, r);
    else if (a.experts <= 128) rank_tokens<4>(a, r);
    else if (a.experts <= 256) rank_tokens<8>(a, r);
    else rank_tokens<16>(a, r);
    __syncthreads();
    if (warp == 0) {                                           // rows of h by expert, and the blocks of those that anyone chose
        int rows = 0, n = 0;
        for (int e0 = 0; e0 < a.experts; e0 += 32) {
            const int e = e0 + lane, c = e < a.experts ? __popcll(r.chosen[e]) : 0, b = (c + TOKENS - 1) / TOKENS;
            int upto = c << 16 | b;                            // both running sums at once (each at most 512)
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const int u = __shfl_up_sync(~0u, upto, o);
                if (lane >= o) upto += u;
            }
            const int row = rows + (upto >> 16) - c, block = n + (upto & 0xffff) - b;
            if (e < a.experts) r.first[e] = (short)row;
            for (int i = 0; i < b; ++i)
                r.blocks[block + i] = Block{(short)e, (short)(row + i * TOKENS), (short)min(TOKENS, c - i * TOKENS)};
            const int all = __shfl_sync(~0u, upto, 31);
            rows += all >> 16;
            n += all & 0xffff;
        }
        if (lane == 0) r.n_blocks = n;
    }
    __syncthreads();
    for (int t = warp; t < a.tokens; t += WARPS)
        if (lane < a.top_k) {
            const int e = r.ids[t][lane], row = r.first[e] + __popcll(r.chosen[e] & ((1ull << t) - 1));
            r.token[row] = (unsigned char)t;
            r.row[t][lane] = (short)row;
        }
    __syncthreads();
}

// x of `count` tokens (token(i): which), columns of `tiles` tiles from tile `first` on -> operand terms [terms][count][ld] in the order of place_of
template <int DTYPE, typename TOKEN>
__device__ __forceinline__ void stage_tokens(const MoeArgs &a, uint16_t *to, int count, int first, int tiles, int ld, TOKEN token) {
    constexpr int TERMS = Operand<DTYPE>::TERMS;
    const int per_token = tiles * (W4_COLS / 8), all = count * per_token;
    for (int i0 = threadIdx.x; i0 < all; i0 += 4 * THREADS) {
        Raw8<DTYPE> v[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int i = min(i0 + j * THREADS, all - 1), n = i / per_token;
            v[j] = load_x8<DTYPE>(static_cast<const typename Element<DTYPE>::type *>(a.x) + token(n) * a.x_stride, first * W4_COLS + (i - n * per_token) * 8,
                                  a.hidden, a.wide);
        }
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int i = min(i0 + j * THREADS, all - 1), n = i / per_token, k = (i - n * per_token) * 8;
            uint32_t b[TERMS][4];
            expand_x8<DTYPE, TERMS>(v[j], b);
#pragma unroll
            for (int q = 0; q < TERMS; ++q) {
                uint16_t *row = to + (q * count + n) * ld;
                *reinterpret_cast<uint2 *>(row + place_of(k)) = make_uint2(b[q][0], b[q][1]);
                *reinterpret_cast<uint2 *>(row + place_of(k + 4)) = make_uint2(b[q][2], b[q][3]);
            }
        }
    }
}

// ---- stage 2: h = silu(G x) * (U x)
template <int DTYPE, int PER>
__device__ void expand_stage(const MoeArgs &a, Routing &r, TileRing<SLOTS> &ring, Part &part, Sums &sums, uint16_t *staged) {
    using Op = Operand<DTYPE>;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, g = lane >> 2, t = lane & 3;
    const TokenScales none{0, 0, 0};
    const int row_tiles = a.gate.row_tiles, col_tiles = a.gate.col_tiles, all = r.n_blocks * row_tiles;      // unit = block * row_tiles + row
    const int u0 = (int)((long long)all * blockIdx.x / gridDim.x), u1 = (int)((long long)all * (blockIdx.x + 1) / gridDim.x);
    if (u0 == u1) return;
    const bool chunked = a.chunk_tiles < col_tiles;
    // a run ends with the block where x is staged by block, and after BATCH rows where it is staged in chunks
    auto run_end = [&](int s0) { return a.resident ? u1 : min(u1, min((s0 / row_tiles + 1) * row_tiles, chunked ? s0 + BATCH : u1)); };
    const int ld = a.chunk_tiles * W4_COLS + 32;
    const long long h_plane = (long long)a.tokens * a.top_k * a.h_cols;

    // where the loads are: run, chunk, position in the stretch
    int f_run = u0, f_chunk = 0, f_kt = 0, f_tiles = 0, f_left = 0, f_unit = 0;
    TileSource<true> next = {};
    auto point = [&]() {
        const int b = f_unit / row_tiles, row = f_unit - b * row_tiles;
        const long long e = r.blocks[b].expert;
        next = ring.source_of_both(a.gate, a.gate.base + e * a.gate.matrix_bytes, a.up, a.up.base + e * a.up.matrix_bytes, row, row, f_chunk + f_kt);
    };
    auto locate = [&]() {
        for (; f_run < u1; f_run = run_end(f_run)) {
            for (; f_chunk < col_tiles; f_chunk += a.chunk_tiles) {
                f_tiles = min(a.chunk_tiles, col_tiles - f_chunk);
                const Stretch s((run_end(f_run) - f_run) * f_tiles, WARPS, warp);
                f_left = s.end - s.first;
                if (f_left == 0) continue;
                f_unit = f_run + s.first / f_tiles;
                f_kt = s.first % f_tiles;
                return point();
            }
            f_chunk = 0;
        }
        f_left = 0;
    };
    locate();
    auto fetch = [&]() {
        if (f_left == 0) return ring.close();
        ring.push(next, 1);
        if (--f_left == 0) {
            f_chunk += a.chunk_tiles;
            locate();
        } else if (++f_kt == f_tiles) {
            f_kt = 0;
            ++f_unit;
            point();
        }
    };
#pragma unroll
    for (int i = 0; i < SLOTS - 1; ++i) fetch();

    // G and U sums of an entry of a unit -> h
    auto finish = [&](int unit, int at, int in_tile, float gv, float uv) {
        const int b = unit / row_tiles;
        store_terms(a.h_planes + (long long)(r.blocks[b].first_row + at) * a.h_cols + place_of((unit - b * row_tiles) * W4_ROWS + in_tile), h_plane,
                                    gv / (1.0f + expf(-gv)) * uv);
    };
    for (int run = u0; run < u1; run = run_end(run)) {
        const int n_rows = run_end(run) - run, run_block = run / row_tiles;
        const int count = a.resident ? a.tokens : r.blocks[run_block].rows;        // staged tokens
        for (int chunk = 0; chunk < col_tiles; chunk += a.chunk_tiles) {
            const int tiles = min(a.chunk_tiles, col_tiles - chunk), total = n_rows * tiles;
            if (!a.resident && (chunked || run == u0 || run % row_tiles == 0)) {
                stage_tokens<DTYPE>(a, staged, count, chunk, tiles, ld, [&](int i) { return (int)r.token[r.blocks[run_block].first_row + i]; });
                __syncthreads();
            }
            const Stretch mine(total, WARPS, warp);
            for (int at = mine.first, row = mine.first / tiles; at < mine.end; ++row) {
                const int kt0 = at - row * tiles, n = min(tiles - kt0, mine.end - at);
                const Block block = r.blocks[(run + row) / row_tiles];
                const int token = min(g, block.rows - 1);                          // one that is not there reads the last one's; its sums are not used
                SharedTokens<Op::TERMS> x;
                x.plane = (uint32_t)count * ld * 2;
                x.row = (uint32_t)__cvta_generic_to_shared(staged + (a.resident ? (int)r.token[block.first_row + token] : token) * ld + 8 * t) + kt0 * (W4_COLS * 2);
                float gs[4] = {}, us[4] = {};
                for (int kt = kt0; kt < kt0 + n; ++kt) {
                    const uint32_t slot = ring.pop();
                    const LoadedTokens<Op::TERMS> now(x);
                    multiply_tile<Op::BF16, false, PER, Op::TERMS>(a.gate, ring.slot, slot, 0, now, kt, none, 0, gs);
                    multiply_tile<Op::BF16, false, PER, Op::TERMS>(a.up, ring.slot, slot, 1, now, kt, none, 0, us);
                    fetch();
                    x.row += W4_COLS * 2;
                }
                if (n == tiles && !chunked) {
#pragma unroll
                    for (int q = 0; q < 4; ++q)
                        if (2 * t + (q & 1) < block.rows) finish(run + row, 2 * t + (q & 1), g + 8 * (q >> 1), gs[q], us[q]);
                } else {
                    const bool whole = n == tiles;
                    float (*to)[TOKENS][LD] = whole ? sums.v[row] : part.v[warp][at != mine.first];
#pragma unroll
                    for (int q = 0; q < 4; ++q) {
                        float &gv = to[0][2 * t + (q & 1)][g + 8 * (q >> 1)], &uv = to[1][2 * t + (q & 1)][g + 8 * (q >> 1)];
                        gv = whole && chunk ? gv + gs[q] : gs[q];
                        uv = whole && chunk ? uv + us[q] : us[q];
                    }
                }
                at += n;
            }
            __syncthreads();
            const bool last = chunk + tiles == col_tiles;
            for (int row = warp; row < n_rows; row += WARPS) {                     // rows that several warps share; with chunks, all of them
                const int first = row * tiles, end = first + tiles, p0 = stretch_of(total, WARPS, first);
                const bool whole = Stretch(total, WARPS, p0).end >= end;
                if (whole && (!chunked || !last)) continue;
                for (int i = lane; i < r.blocks[(run + row) / row_tiles].rows * W4_ROWS; i += 32) {
                    const int in_tile = i & 15, at = i >> 4;
                    float gv = 0.0f, uv = 0.0f;
                    if (chunked && (whole || chunk)) { gv = sums.v[row][0][at][in_tile]; uv = sums.v[row][1][at][in_tile]; }
                    if (!whole)
                        for (int p = p0; p < WARPS; ++p) {
                            const Stretch s(total, WARPS, p);
                            if (s.first >= end) break;
                            if (s.end == s.first) continue;
                            gv += part.v[p][s.first < first][0][at][in_tile];
                            uv += part.v[p][s.first < first][1][at][in_tile];
                        }
                    if (last) finish(run + row, at, in_tile, gv, uv);
                    else { sums.v[row][0][at][in_tile] = gv; sums.v[row][1][at][in_tile] = uv; }
                }
            }
            __syncthreads();
        }
    }
}

// ---- stage 3: y = sum of share * D h, ROWS row tiles at a time.  `meet` (the barrier before the stage) is called once the
// first tiles are on their way.  Where D has fewer rows than there are CTAs, `splits` of them share a unit's tiles and leave their part
// of y in the workspace; returns whether that is so (then the parts are still to be added).
template <int PER, int ROWS, typename MEET>
__device__ int combine_stage(const MoeArgs &a, Routing &r, TileRing<SLOTS> &ring, float *shared, MEET meet) {
    constexpr int TERMS = H_TERMS;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, g = lane >> 2, t = lane & 3;
    const TokenScales none{0, 0, 0};
    const int pairs = a.tokens * a.top_k, tiles = a.down.col_tiles, total = r.n_blocks * tiles, units = (a.down.row_tiles + ROWS - 1) / ROWS;
    const long long h_plane = (long long)pairs * a.h_cols;
    float *by_row = shared;                                                        // [ROWS][pairs][LD]
    DownPart<ROWS> &part = *reinterpret_cast<DownPart<ROWS> *>(shared + ROWS * pairs * LD);

    // at least MIN_TILES tiles for each of the CTAs that share a unit: the parts cost a further barrier
    constexpr int MIN_TILES = 96;
    const int splits = max(1, min(min((int)gridDim.x / units, MAX_SPLITS), ROWS * total / MIN_TILES)), split = blockIdx.x / units;
    const int unit0 = splits == 1 ? blockIdx.x : split < splits ? blockIdx.x - split * units : units, unit_step = splits == 1 ? gridDim.x : units;
    const Stretch mine(total, WARPS * splits, splits == 1 ? warp : min(split, splits - 1) * WARPS + warp);
    const int my_first = Stretch(total, splits, splits == 1 ? 0 : min(split, splits - 1)).first, my_end = Stretch(total, splits, splits == 1 ? 0 : min(split, splits - 1)).end;
    int f_unit = unit0, f_b = 0, f_kt = 0, f_left = 0;                        // where the loads are
    TileSource<ROWS == 2> next = {};
    auto point = [&]() {
        const uint8_t *m = a.down.base + r.blocks[min(f_b, r.n_blocks - 1)].expert * a.down.matrix_bytes;
        if constexpr (ROWS == 2) next = ring.source_of_both(a.down, m, a.down, m, f_unit * 2, min(f_unit * 2 + 1, a.down.row_tiles - 1), f_kt);
        else next = ring.template source<false>(a.down, m, f_unit, f_kt);
    };
    auto locate = [&]() {
        f_left = f_unit < units ? mine.end - mine.first : 0;
        f_b = f_left ? mine.first / tiles : 0;
        f_kt = mine.first - f_b * tiles;
        if (f_left) point();
    };
    locate();
    auto fetch = [&]() {
        if (f_left == 0) return ring.close();
        const int n = ROWS == 2 ? 1 : min(2, min(f_left, tiles - f_kt));
        ring.push(next, n);
        f_left -= n;
        f_kt += n;
        if (f_left == 0) {
            f_unit += unit_step;
            locate();
        } else if (f_kt == tiles) {
            f_kt = 0;
            ++f_b;
            point();
        }
    };
#pragma unroll
    for (int i = 0; i < SLOTS - 1; ++i) fetch();
    meet();

    for (int unit = unit0; unit < units; unit += unit_step) {
        for (int at = mine.first; at < mine.end;) {
            const int b = at / tiles, kt0 = at - b * tiles, n = min(tiles - kt0, mine.end - at);
            const Block block = r.blocks[b];
            GlobalTokens<TERMS> x;                          // a token that is not there reads the last one's row; its sums are not used
            x.plane = h_plane;
            x.row = a.h_planes + (long long)(block.first_row + min(g, block.rows - 1)) * a.h_cols + 8 * t + kt0 * W4_COLS;
            float s[ROWS][4] = {};
            uint32_t slot = 0;
            if (ROWS == 2) {
                for (int kt = kt0; kt < kt0 + n; ++kt) {
                    const LoadedTokens<TERMS> now(x);
                    slot = ring.pop();
                    multiply_tile<true, false, PER, TERMS>(a.down, ring.slot, slot, 0, now, kt, none, 0, s[0]);
                    multiply_tile<true, false, PER, TERMS>(a.down, ring.slot, slot, 1, now, kt, none, 0, s[ROWS - 1]);
                    fetch();
                    x.row += W4_COLS;
                }
            } else {
                for (int kt = kt0; kt < kt0 + n; ++kt) {       // (a tile's h loads are all under way before the first is used)
                    const LoadedTokens<TERMS> now(x);
                    const int which = (kt - kt0) & 1;
                    if (!which) slot = ring.pop();
                    multiply_tile<true, false, PER, TERMS>(a.down, ring.slot, slot, which, now, kt, none, 0, s[0]);
                    if (which || kt + 1 == kt0 + n) fetch();
                    x.row += W4_COLS;
                }
            }
#pragma unroll
            for (int m = 0; m < ROWS; ++m) {
                float *to = n == tiles ? by_row + (m * pairs + block.first_row) * LD : &part.v[warp][at != mine.first][m][0][0];
#pragma unroll
                for (int q = 0; q < 4; ++q)
                    if (n != tiles || 2 * t + (q & 1) < block.rows) to[(2 * t + (q & 1)) * LD + g + 8 * (q >> 1)] = s[m][q];
            }
            at += n;
        }
        __syncthreads();
        for (int b = warp; b < r.n_blocks; b += WARPS) {       // blocks that several warps share, or of which this CTA has a part, or none
            const int first = b * tiles, end = first + tiles, from = max(first, my_first), to = min(end, my_end);
            int p0 = WARPS * splits;
            if (from < to) {
                p0 = stretch_of(total, WARPS * splits, from);
                const Stretch s(total, WARPS * splits, p0);
                if (s.first <= first && s.end >= end) continue;
            }
            const Block block = r.blocks[b];
            for (int m = 0; m < ROWS; ++m)
                for (int i = lane; i < block.rows * W4_ROWS; i += 32) {
                    float v = 0.0f;
                    for (int p = p0; p < WARPS * splits; ++p) {
                        const Stretch s(total, WARPS * splits, p);
                        if (s.first >= to) break;
                        if (s.end > s.first) v += part.v[p % WARPS][s.first < first][m][i >> 4][i & 15];
                    }
                    by_row[(m * pairs + block.first_row + (i >> 4)) * LD + (i & 15)] = v;
                }
        }
        __syncthreads();
        for (int i = threadIdx.x; i < a.tokens * W4_ROWS * ROWS; i += THREADS) {
            const int in_tile = i & 15, m = ROWS == 2 ? (i >> 4) & 1 : 0, token = i >> (ROWS == 2 ? 5 : 4), row = (unit * ROWS + m) * W4_ROWS + in_tile;
            float v = 0.0f;
            for (int j = 0; j < a.top_k; ++j) v = fmaf(r.shares[token][j], by_row[(m * pairs + r.row[token][j]) * LD + in_tile], v);
            if (row >= a.hidden) continue;
            if (!r.fine) v = __int_as_float(0x7fffffff);
            if (splits > 1) a.parts[((long long)split * a.tokens + token) * a.hidden + row] = v;
            else store_from_float(a.y, token * a.y_stride + row, a.dtype, v);
        }
        __syncthreads();
    }
    return splits;
}

template <typename T, int DTYPE, int PER>
__global__ void __launch_bounds__(THREADS, 1) moe_kernel(const MoeArgs a) {
    extern __shared__ __align__(16) uint8_t shared[];
    Routing &r = *reinterpret_cast<Routing *>(shared);
    const int ring_bytes = SLOTS * slot_layout(a.gate).bytes, warp = threadIdx.x >> 5;
    uint8_t *rings = shared + sizeof(Routing), *rest = rings + WARPS * ring_bytes;
    const bool chunked = a.chunk_tiles < a.gate.col_tiles;
    Part &part = *reinterpret_cast<Part *>(rest);
    Sums &sums = *reinterpret_cast<Sums *>(rest + sizeof(Part));
    uint16_t *staged = reinterpret_cast<uint16_t *>(rest + sizeof(Part) + (chunked ? sizeof(Sums) : 0));

    unsigned long long begun = 0;                              // what earlier launches left the count at
    if (threadIdx.x == 0) {
        asm volatile("ld.relaxed.gpu.global.u64 %0, [%1];" : "=l"(begun) : "l"(a.arrivals) : "memory");
        begun -= (begun & COUNT) % gridDim.x;
        r.fine = 1;
    }
    if constexpr (DTYPE == MOM_F32) {
        route_fma<T, float>(a, *reinterpret_cast<Slots *>(rest));
    } else {
        if (a.router_dtype == MOM_F32) route_fma<T, float>(a, *reinterpret_cast<Slots *>(rest));
        else route_mma<DTYPE>(a, *reinterpret_cast<Slots *>(rest));
    }
    for (int e = threadIdx.x; e < a.experts; e += THREADS) r.chosen[e] = 0;
    grid_arrive(a, r);
    fill_planes(a);                                     // (what follows needs no other CTA's logits)
    if (a.resident) stage_tokens<DTYPE>(a, staged, a.tokens, 0, a.gate.col_tiles, a.chunk_tiles * W4_COLS + 32, [](int i) { return i; });
    grid_wait(a, r, begun, 1);                                    // (given up: the next barrier says so to all)
    rank_experts(a, r);

    TileRing<SLOTS> ring((uint32_t)__cvta_generic_to_shared(rings + warp * ring_bytes), a.gate);
    expand_stage<DTYPE, PER>(a, r, ring, part, sums, staged);

    // all of stage 2's slots have been used (a CTA with nothing to do has filled none): only empty groups lie behind, the ring starts anew (D's
    // group size and types are G's)
    __syncthreads();
    asm volatile("cp.async.wait_all;" ::: "memory");
    ring.tail = ring.head;
    grid_arrive(a, r);
    auto meet = [&]() { grid_wait(a, r, begun, 2); };
    const int splits = a.pair_rows ? combine_stage<PER, 2>(a, r, ring, reinterpret_cast<float *>(rest), meet)
                                   : combine_stage<PER, 1>(a, r, ring, reinterpret_cast<float *>(rest), meet);
    // (every CTA arrives three times, so that the count stays a multiple of the grid)
    grid_arrive(a, r);
    if (splits == 1) return;
    grid_wait(a, r, begun, 3);
    for (long long i = (long long)blockIdx.x * THREADS + threadIdx.x; i < (long long)a.tokens * a.hidden; i += (long long)gridDim.x * THREADS) {
        float v = 0.0f;
        for (int p = 0; p < splits; ++p) v += a.parts[(long long)p * a.tokens * a.hidden + i];
        if (!r.fine) v = __int_as_float(0x7fffffff);
        store_from_float(a.y, i / a.hidden * a.y_stride + i % a.hidden, a.dtype, v);
    }
}

size_t logits_bytes(const mom_moe_desc_t &d, int64_t tokens) { return align_up((size_t)tokens * d.experts * 4, WS_ALIGN); }

size_t parts_bytes(const mom_moe_desc_t &d, int64_t tokens) { return align_up((size_t)MAX_SPLITS * tokens * d.hidden * 4, WS_ALIGN); }
size_t h_bytes(const mom_moe_desc_t &d, int64_t tokens) {
    return align_up((size_t)H_TERMS * tokens * d.top_k * align_up((size_t)d.inner, W4_COLS) * 2, WS_ALIGN);
}

template <typename T, int DTYPE, int PER>
cudaError_t launch(MoeArgs a, int sm_count, cudaStream_t stream) {
    cudaError_t e = raise_smem_limit<moe_kernel<T, DTYPE, PER>>(SHARED_LIMIT);
    if (e != cudaSuccess) return e;
    // x of all tokens stays in shared memory if it fits, else the tokens of one block at a time do, else (wide layers) chunks of their columns
    const int fixed = (int)sizeof(Routing) + WARPS * SLOTS * slot_layout(a.gate).bytes, room = SHARED_LIMIT - fixed - (int)sizeof(Part);
    constexpr int ENTRY = 2 * Operand<DTYPE>::TERMS;           // bytes of an entry of x
    static_assert(SHARED_LIMIT - (int)sizeof(Routing) - WARPS * SLOTS * MAX_SLOT_BYTES - (int)sizeof(Part) - (int)sizeof(Sums) >= TOKENS * ENTRY * (W4_COLS + 32), "room for a tile");
    const long long row = a.gate.col_tiles * W4_COLS + 32;
    a.chunk_tiles = a.gate.col_tiles;
    a.resident = a.tokens * row * ENTRY <= room;
    if (!a.resident && TOKENS * row * ENTRY > room) {
        const int most = ((room - (int)sizeof(Sums)) / (TOKENS * ENTRY) - 32) / W4_COLS, chunks = (a.gate.col_tiles + most - 1) / most;
        a.chunk_tiles = (a.gate.col_tiles + chunks - 1) / chunks;
    }
    // two row tiles of D at a time where every CTA gets some and the results fit
    const int pairs = a.tokens * a.top_k;
    a.pair_rows = a.down.row_tiles > sm_count && fixed + 2 * pairs * LD * 4 + (int)sizeof(DownPart<2>) <= SHARED_LIMIT;
    static_assert(sizeof(Routing) + WARPS * SLOTS * MAX_SLOT_BYTES + MAX_PAIRS * LD * 4 + sizeof(DownPart<1>) <= SHARED_LIMIT, "room for stage 3");
    void *args[] = {&a};
    return cudaLaunchCooperativeKernel(reinterpret_cast<const void *>(moe_kernel<T, DTYPE, PER>), dim3(sm_count), dim3(THREADS), args, SHARED_LIMIT, stream);
}

template <typename T, int DTYPE>
cudaError_t launch(const MoeArgs &a, int per, int sm_count, cudaStream_t stream) {
    return per == 1 ? launch<T, DTYPE, 1>(a, sm_count, stream) : per == 2 ? launch<T, DTYPE, 2>(a, sm_count, stream) : launch<T, DTYPE, 4>(a, sm_count, stream);
}

}  // namespace

}  // namespace mom

extern "C" {

mom_status_t mom_moe_plan(const mom_moe_desc_t *d, mom_moe_plan_t **out_plan) {
    using namespace mom;
    if (!d || !out_plan || d->experts < 1 || d->top_k < 1 || d->top_k > d->experts || (d->renormalize != 0 && d->renormalize != 1)) return MOM_ERR_INVALID_ARG;
    if (!is_float_type(d->dtype) || (d->router_dtype != d->dtype && d->router_dtype != MOM_F32)) return MOM_ERR_DTYPE;
    mom_w4_desc_t gate{d->inner, d->hidden, d->experts, d->group, d->scale_dtype, d->zeros}, down = gate;
    down.rows = d->hidden;
    down.cols = d->inner;
    mom_status_t st = check_w4_desc(&gate);
    if (st == MOM_OK) st = check_w4_desc(&down);
    if (st != MOM_OK) return st;
    if (d->experts > MAX_E || d->top_k > MAX_K || d->hidden > MAX_WIDTH || d->inner > MAX_WIDTH) return MOM_ERR_LIMIT;
    mom_moe_plan_t *p = new (std::nothrow) mom_moe_plan_t();
    if (!p) return MOM_ERR_ALLOC;
    p->desc = *d;
    p->gate = gate;
    p->down = down;
    *out_plan = p;
    return MOM_OK;
}

mom_status_t mom_moe_plan_destroy(mom_moe_plan_t *plan) {
    if (plan && plan->block) cudaFree(plan->block);
    delete plan;
    return MOM_OK;
}

mom_status_t mom_moe_workspace_bytes(const mom_moe_plan_t *plan, int64_t tokens, size_t *bytes) {
    using namespace mom;
    if (!plan || !bytes || tokens < 0) return MOM_ERR_INVALID_ARG;
    if (tokens > MAX_T) return MOM_ERR_LIMIT;
    if (tokens * plan->desc.top_k > MAX_PAIRS) return MOM_ERR_LIMIT;
    *bytes = logits_bytes(plan->desc, tokens) + h_bytes(plan->desc, tokens) + parts_bytes(plan->desc, tokens);
    return MOM_OK;
}

mom_status_t mom_moe_execute(const mom_moe_plan_t *plan, int64_t tokens, const void *x, int64_t x_stride, const void *router, const void *gate,
                             const void *up, const void *down, void *y, int64_t y_stride, int32_t *expert_ids, float *shares, void *workspace,
                             size_t workspace_bytes, mom_stream_t stream) {
    using namespace mom;
    size_t need = 0;
    const mom_status_t sized = mom_moe_workspace_bytes(plan, tokens, &need);
    if (sized != MOM_OK) return sized;
    const mom_moe_desc_t &d = plan->desc;
    if ((x_stride != 0 && x_stride < d.hidden) || (y_stride != 0 && y_stride < d.hidden)) return MOM_ERR_INVALID_ARG;
    if (tokens == 0) return MOM_OK;
    if (!x || !router || !gate || !up || !down || !y || !workspace) return MOM_ERR_INVALID_ARG;
    const int bytes = element_bytes(d.dtype);
    if (!aligned_to(x, bytes) || !aligned_to(y, bytes) || !aligned_to(router, element_bytes(d.router_dtype)) || !aligned_to(gate, WS_ALIGN) ||
        !aligned_to(up, WS_ALIGN) || !aligned_to(down, WS_ALIGN) || !aligned_to(expert_ids, 4) || !aligned_to(shares, 4) || !aligned_to(workspace, WS_ALIGN))
        return MOM_ERR_ALIGNMENT;
    if (workspace_bytes < need) return MOM_ERR_WORKSPACE_TOO_SMALL;
    int device = 0, sm_count = 0;
    const int st = current_sm100(&device, &sm_count);
    if (st != MOM_OK) return (mom_status_t)st;

    std::lock_guard<std::mutex> lock(plan->mutex);
    if (plan->device != device) {
        if (plan->block) cudaFree(plan->block);
        plan->block = nullptr;
        plan->device = -1;
        if (cudaMalloc(&plan->block, 64) != cudaSuccess) return MOM_ERR_ALLOC;
        // (on the caller's stream: the kernel that follows there must find it cleared, and other streams need not wait for the default one)
        if (cudaMemsetAsync(plan->block, 0, 64, stream) != cudaSuccess) return MOM_ERR_CUDA;
        plan->device = device;
    }
    MoeArgs a;
    a.gate = w4_view(plan->gate, gate);
    a.up = w4_view(plan->gate, up);
    a.down = w4_view(plan->down, down);
    a.x = x; a.router = router; a.y = y;
    a.x_stride = x_stride ? x_stride : d.hidden;
    a.y_stride = y_stride ? y_stride : d.hidden;
    a.tokens = (int)tokens; a.hidden = (int)d.hidden; a.inner = (int)d.inner; a.experts = d.experts; a.top_k = d.top_k;
    a.renormalize = d.renormalize; a.dtype = d.dtype; a.router_dtype = d.router_dtype;
    a.wide = aligned_to(x, 16) && (a.x_stride * bytes) % 16 == 0;
    const int per = stretches_per_scale(d.group, 0);
    a.logits = static_cast<float *>(workspace);
    a.h_planes = reinterpret_cast<uint16_t *>(static_cast<uint8_t *>(workspace) + logits_bytes(d, tokens));
    a.parts = reinterpret_cast<float *>(static_cast<uint8_t *>(workspace) + logits_bytes(d, tokens) + h_bytes(d, tokens));
    a.h_cols = (int)align_up((size_t)d.inner, W4_COLS);
    a.ids = expert_ids; a.shares = shares;
    a.arrivals = plan->block;
    a.status = reinterpret_cast<int32_t *>(plan->block + 1);
    a.missing = plan->probe_ns != 0;
    a.limit_ns = plan->probe_ns ? plan->probe_ns : WAIT_LIMIT_NS;
    plan->probe_ns = 0;
    cudaError_t e;
    if (d.dtype == MOM_F32) e = launch<float, MOM_F32>(a, per, sm_count, stream);
    else if (d.dtype == MOM_BF16) e = launch<__nv_bfloat16, MOM_BF16>(a, per, sm_count, stream);
    else e = launch<__half, MOM_F16>(a, per, sm_count, stream);
    return e == cudaSuccess ? MOM_OK : MOM_ERR_CUDA;
}

mom_status_t mom_moe_device_status(const mom_moe_plan_t *plan, int32_t *code, int32_t *detail) {
    using namespace mom;
    if (!plan || !code) return MOM_ERR_INVALID_ARG;
    std::lock_guard<std::mutex> lock(plan->mutex);
    int32_t host[2] = {0, 0};
    if (plan->block) {
        if (cudaMemcpy(host, plan->block + 1, sizeof(host), cudaMemcpyDeviceToHost) != cudaSuccess) return MOM_ERR_CUDA;
        if (host[0] != 0 && !cleared(plan->block, 64)) return MOM_ERR_CUDA;
    }
    *code = host[0];
    if (detail) *detail = host[1];
    return MOM_OK;
}

mom_status_t mom_moe_probe_wait_timeout(const mom_moe_plan_t *plan, double limit_ms) {
    if (!plan || !(limit_ms > 0.0) || limit_ms > 1000.0) return MOM_ERR_INVALID_ARG;
    std::lock_guard<std::mutex> lock(plan->mutex);
    plan->probe_ns = (unsigned long long)(limit_ms * 1.0e6) + 1;
    return MOM_OK;
}

}  // extern "C"
