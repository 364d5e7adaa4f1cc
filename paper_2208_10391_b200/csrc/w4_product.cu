// Y = X * W^T (+ T) with W in the 4-bit container, for up to eight tokens.
//
// One persistent CTA of 16 warps per SM takes a run of neighbouring 16-row tiles of W; where x is large against W's share of a CTA, a
// cluster of up to four CTAs takes the run and each of them a part of the columns.  The tokens of x are staged in shared
// memory once, as operand terms (16 bits, f32 in three), whole or in chunks of columns where they do not fit.  The run's 16 x 128
// tiles, row by row, are one sequence that is cut into 16 even stretches, one per warp: a warp streams its tiles through its own ring
// (w4.cuh), multiplies them on mma.sync and only at the end of a row puts its f32 sums away.  A row that lies wholly in one stretch
// is finished by its warp; the (at most two) rows that it shares with its neighbours go to slots that are added in the
// warps' order once all have arrived, and the cluster's sums are added in its CTAs' order: the same bits every time.
// Measured: 1 token, 28672 x 8192 bf16 30.5 us (121 MB: 4.0 TB/s of the 6.5 that a copy reaches; 174 warp instructions per tile at 2.65 a
// cycle bound it, 24 warps or a smaller ring change nothing); 1 x 1024 x 1024 3.5 us (a launch); 7 x 1999 x 5003 in f32 11.8 us;
// with 8-bit tokens 1 x 28672 x 8192 30.0 us in e4m3 and in int8, 8 x 28672 x 8192 in e4m3 37 us.
#include <algorithm>

#include <cooperative_groups.h>

#include "device_common.cuh"
#include "tc_ptx.cuh"
#include "w4_product.h"

namespace mom {

namespace {

namespace cg = cooperative_groups;

constexpr int WARPS = 16, SLOTS = 3;

constexpr int BATCH = 16;                              // row tiles of a run
struct ProductShared {
    float part[WARPS][2][8][W4_ROWS + 1];         // a stretch's first and last row, where it has only a part of them
    float sums[BATCH][8][W4_ROWS + 1];
    struct { short first_warp, end_warp, first_slot; } shared_by[BATCH];   // end_warp 0: the row lies in one stretch
};
constexpr int SHARED_LIMIT = 227 * 1024;
// the rings follow, then x: [terms][tokens][chunk columns + 32] (rows 64 bytes off each other's banks), and the scales of 8-bit tokens
__host__ __device__ inline int chunk_scales(int tiles, int x_group_shift) { return ((tiles * W4_COLS - 1) >> x_group_shift) + 1; }

template <int DTYPE, int PER>
__global__ void __launch_bounds__(WARPS * 32, 1) w4_product_kernel(const W4ProductArgs a) {
    extern __shared__ __align__(16) uint8_t shared[];
    using Op = Operand<DTYPE>;
    ProductShared &sh = *reinterpret_cast<ProductShared *>(shared);
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, g = lane >> 2, t = lane & 3;
    const W4View &w = a.w;
    const uint32_t ring_bytes = SLOTS * slot_layout(w).bytes;
    uint8_t *rings = shared + sizeof(ProductShared);
    uint16_t *staged = reinterpret_cast<uint16_t *>(rings + WARPS * ring_bytes);
    const int ld = a.chunk_tiles * W4_COLS + 32;
    const int tokens = a.tokens;
    const int plane = tokens * ld;
    float *scales = reinterpret_cast<float *>(staged + (long long)Op::TERMS * plane);
    const TokenScales xs{(uint32_t)__cvta_generic_to_shared(scales), chunk_scales(a.chunk_tiles, a.x_group_shift), a.x_group_shift};
    // a token that is not there reads the last one's row; its sums are not used
    const uint32_t my_row = (uint32_t)__cvta_generic_to_shared(staged + min(g, tokens - 1) * ld + 8 * t);

    const int teams = gridDim.x / a.split, team = blockIdx.x / a.split, rank = blockIdx.x - team * a.split;
    const int rt_first = (int)((long long)w.row_tiles * team / teams), rt_end = (int)((long long)w.row_tiles * (team + 1) / teams);
    const int ct_first = rank * a.part_tiles, ct_end = min(ct_first + a.part_tiles, w.col_tiles);      // (may be empty)

    // where the loads are: run, chunk, position in the stretch
    TileRing<SLOTS> ring((uint32_t)__cvta_generic_to_shared(rings + warp * ring_bytes), w);
    int f_run = rt_first, f_chunk = ct_first, f_kt = 0, f_tiles = 0, f_left = 0;
    TileSource<false> next = ring.source<false>(w, w.base, rt_first, 0);
    int f_row = rt_first;
    auto locate = [&]() {                                      // the first tile of the stretch, of the next chunk and run that has one
        for (; f_run < rt_end; f_run += BATCH) {
            for (; f_chunk < ct_end; f_chunk += a.chunk_tiles) {
                f_tiles = min(a.chunk_tiles, ct_end - f_chunk);
                const Stretch s(min(BATCH, rt_end - f_run) * f_tiles, WARPS, warp);
                f_left = s.end - s.first;
                if (f_left == 0) continue;
                f_row = f_run + s.first / f_tiles;
                f_kt = s.first % f_tiles;
                next = ring.source<false>(w, w.base, f_row, f_chunk + f_kt);
                return;
            }
            f_chunk = ct_first;
        }
        f_left = 0;
    };
    locate();
    allow_dependents();
    grid_dependency_wait();                                    // nothing has been read yet
    auto fetch = [&]() {
        if (f_left == 0) return ring.close();
        const int n = min(2, min(f_left, f_tiles - f_kt));
        ring.push(next, n);
        f_left -= n;
        f_kt += n;
        if (f_left == 0) {
            f_chunk += a.chunk_tiles;
            locate();
        } else if (f_kt == f_tiles) {
            f_kt = 0;
            next = ring.source<false>(w, w.base, ++f_row, f_chunk);
        }
    };
#pragma unroll
    for (int i = 0; i < SLOTS - 1; ++i) fetch();

    for (int run = rt_first; run < rt_end; run += BATCH) {
        const int n_rows = min(BATCH, rt_end - run);
        for (int chunk = ct_first; chunk < ct_end; chunk += a.chunk_tiles) {
            const int tiles = min(a.chunk_tiles, ct_end - chunk);
            if (a.chunk_tiles < a.part_tiles || run == rt_first) {
                // eight entries a thread, four times at once: what costs here is waiting for the loads
                const int per_token = tiles * (W4_COLS / 8), all = tokens * per_token;
                for (int i0 = threadIdx.x; i0 < all; i0 += 4 * WARPS * 32) {
                    Raw8<DTYPE> v[4];
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const int i = min(i0 + j * WARPS * 32, all - 1), token = i / per_token, k = (i - token * per_token) * 8;
                        v[j] = load_x8<DTYPE>(static_cast<const typename Element<DTYPE>::type *>(a.x) + token * a.x_stride,
                                              chunk * W4_COLS + k, w.cols, a.wide);
                    }
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const int i = min(i0 + j * WARPS * 32, all - 1), token = i / per_token, k = (i - token * per_token) * 8;
                        uint32_t b[Op::TERMS][4];
                        expand_x8<DTYPE, Op::TERMS>(v[j], b);
#pragma unroll
                        for (int s = 0; s < Op::TERMS; ++s)
                        {
                            uint16_t *to = staged + s * plane + token * ld;
                            *reinterpret_cast<uint2 *>(to + place_of(k)) = make_uint2(b[s][0], b[s][1]);
                            *reinterpret_cast<uint2 *>(to + place_of(k + 4)) = make_uint2(b[s][2], b[s][3]);
                        }
                    }
                }
                if (Op::EIGHT) {                               // the tokens' scales of the chunk
                    for (int i = threadIdx.x; i < tokens * xs.stride; i += WARPS * 32) {
                        const int token = i / xs.stride, group = min(((chunk * W4_COLS) >> a.x_group_shift) + i - token * xs.stride, a.x_groups - 1);
                        scales[i] = a.x_scales[(long long)token * a.x_groups + group];
                    }
                }
                __syncthreads();
            }
            const int all = n_rows * tiles;
            const Stretch mine(all, WARPS, warp);
            if (threadIdx.x < n_rows) {
                const int first = threadIdx.x * tiles, p = stretch_of(all, WARPS, first);
                const bool whole = Stretch(all, WARPS, p).end >= first + tiles;
                sh.shared_by[threadIdx.x].first_warp = (short)p;
                sh.shared_by[threadIdx.x].first_slot = Stretch(all, WARPS, p).first < first;
                sh.shared_by[threadIdx.x].end_warp = whole ? 0 : (short)(stretch_of(all, WARPS, first + tiles - 1) + 1);
            }
            if (mine.first == mine.end)
                for (int i = lane; i < 8 * (W4_ROWS + 1); i += 32) (&sh.part[warp][0][0][0])[i] = 0.0f;
            for (int at = mine.first, row = mine.first / tiles; at < mine.end; ++row) {
                const int kt0 = at - row * tiles, n = min(tiles - kt0, mine.end - at);
                float sum[4] = {};
                for (int kt = kt0; kt < kt0 + n; kt += 2) {
                    const uint32_t slot = ring.pop();
                    SharedTokens<Op::TERMS> x;
                    x.plane = plane * 2;
                    x.row = my_row + kt * (W4_COLS * 2);
                    multiply_tile<Op::BF16, Op::EIGHT, PER, Op::TERMS>(w, ring.slot, slot, 0, x, kt, xs, tokens, sum);
                    if (kt + 1 < kt0 + n) {
                        x.row += W4_COLS * 2;
                        multiply_tile<Op::BF16, Op::EIGHT, PER, Op::TERMS>(w, ring.slot, slot, 1, x, kt + 1, xs, tokens, sum);
                    }
                    fetch();
                }
                const bool whole = n == tiles;
                float (*to)[W4_ROWS + 1] = whole ? sh.sums[row] : sh.part[warp][at != mine.first];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    float &v = to[2 * t + (i & 1)][g + 8 * (i >> 1)];
                    v = whole && chunk > ct_first ? v + sum[i] : sum[i];
                }
                at += n;
            }
            __syncthreads();
            for (int row = warp; row < n_rows; row += WARPS) {             // the rows that several warps share
                const int p0 = sh.shared_by[row].first_warp, p1 = sh.shared_by[row].end_warp;
                if (!p1) continue;
                for (int i = lane; i < tokens * W4_ROWS; i += 32) {
                    const int r = i & 15, token = i >> 4;
                    float v = chunk > ct_first ? sh.sums[row][token][r] : 0.0f;
                    v += sh.part[p0][sh.shared_by[row].first_slot][token][r];
                    for (int p = p0 + 1; p < p1; ++p) v += sh.part[p][0][token][r];
                    sh.sums[row][token][r] = v;
                }
            }
            __syncthreads();
        }
        // the CTA's rows of the run: all of them, or with a cluster every split-th
        if (a.split > 1) {
            if (ct_first >= ct_end)
                for (int i = threadIdx.x; i < (int)(sizeof(sh.sums) / 4); i += WARPS * 32) (&sh.sums[0][0][0])[i] = 0.0f;
            ptx::cluster_sync();
        }
        for (int row = warp * a.split + rank; row < n_rows; row += WARPS * a.split)
            for (int i = lane; i < tokens * W4_ROWS; i += 32) {
                const int r = i & 15, token = i >> 4, out = (run + row) * W4_ROWS + r;
                if (out >= w.rows) continue;
                float v = 0.0f;
                if (a.split == 1) v = sh.sums[row][token][r];
                else
                    for (int p = 0; p < a.split; ++p) v += *cg::this_cluster().map_shared_rank(&sh.sums[row][token][r], p);
                if (a.add) v += load_as_float(a.add, token * a.add_stride + out, a.y_dtype);
                store_from_float(a.y, token * a.y_stride + out, a.y_dtype, v);
            }
        if (a.split > 1) ptx::cluster_sync();
        else __syncthreads();
    }
}

template <int DTYPE, int PER>
cudaError_t launch(W4ProductArgs a, int sm_count, cudaStream_t stream) {
    cudaError_t e = raise_smem_limit<w4_product_kernel<DTYPE, PER>>(SHARED_LIMIT);
    if (e != cudaSuccess) return e;
    const int fixed = sizeof(ProductShared) + WARPS * SLOTS * slot_layout(a.w).bytes, tokens = a.tokens;                  // at most eight
    const int rows = tokens * Operand<DTYPE>::TERMS;
    const int tile_bytes = W4_COLS * 2 + (Operand<DTYPE>::EIGHT ? 4 * (W4_COLS >> 5) : 0);    // of a token and term, scales included
    const int most = ((SHARED_LIMIT - fixed) / rows - 64) / tile_bytes;                       // tiles of x beside the rest
    static_assert((SHARED_LIMIT - (int)sizeof(ProductShared) - WARPS * SLOTS * MAX_SLOT_BYTES) / (8 * Operand<DTYPE>::TERMS) - 64 >= W4_COLS * 2 + 16, "room for a tile");
    // Columns are split where that saves more staging of x (counted in tiles' worth: a CTA stages about STAGE entries in the time of
    // one tile) than the even deal of rows and the cluster's meeting cost.
    constexpr double STAGE = 600.0 / Operand<DTYPE>::TERMS, MEET = 40.0;
    double best = 0.0;
    a.split = 0;
    int teams = 0;
    for (int split = 1; split <= 4; split *= 2) {
        const int room = split == 1 ? sm_count : resident_clusters<w4_product_kernel<DTYPE, PER>>(split, WARPS * 32, SHARED_LIMIT);
        if (room < 1 || (split > 1 && a.w.col_tiles < 4 * split)) continue;
        const int n = a.w.row_tiles < room ? a.w.row_tiles : room, part = (a.w.col_tiles + split - 1) / split;
        const double tiles = (double)((a.w.row_tiles + n - 1) / n) * part, restage = part > most ? (a.w.row_tiles + n * BATCH - 1) / (n * BATCH) : 1;
        const double cost = tiles + restage * part * W4_COLS * tokens / STAGE + (split > 1 ? MEET : 0.0);
        if (a.split == 0 || cost < best) { best = cost; a.split = split; teams = n; }
    }
    a.part_tiles = (a.w.col_tiles + a.split - 1) / a.split;
    const int chunks = (a.part_tiles + most - 1) / most;
    a.chunk_tiles = (a.part_tiles + chunks - 1) / chunks;
    const int bytes = fixed + rows * (a.chunk_tiles * W4_COLS + 32) * 2 + (Operand<DTYPE>::EIGHT ? tokens * chunk_scales(a.chunk_tiles, a.x_group_shift) * 4 : 0);
    return launch_dependent(w4_product_kernel<DTYPE, PER>, dim3(teams * a.split), dim3(WARPS * 32), bytes, stream, a.split, a);
}

template <int DTYPE>
cudaError_t launch(const W4ProductArgs &a, int per, int sm_count, cudaStream_t stream) {
    return per == 1 ? launch<DTYPE, 1>(a, sm_count, stream) : per == 2 ? launch<DTYPE, 2>(a, sm_count, stream) : launch<DTYPE, 4>(a, sm_count, stream);
}

}  // namespace

cudaError_t launch_w4_product(const W4ProductArgs &a, int x_dtype, int per, int sm_count, cudaStream_t stream) {
    switch (x_dtype) {
        case MOM_F32: return launch<MOM_F32>(a, per, sm_count, stream);
        case MOM_BF16: return launch<MOM_BF16>(a, per, sm_count, stream);
        case MOM_F16: return launch<MOM_F16>(a, per, sm_count, stream);
        case MOM_E4M3: return launch<MOM_E4M3>(a, per, sm_count, stream);
        default: return launch<MOM_INT8>(a, per, sm_count, stream);
    }
}

}  // namespace mom

extern "C" mom_status_t mom_w4_product(const mom_w4_product_desc_t *d, const void *container, const void *x, const float *x_scales,
                                       const void *add, void *y, mom_stream_t stream) {
    using namespace mom;
    if (!d || d->reserved != 0 || d->tokens < 0) return MOM_ERR_INVALID_ARG;
    mom_status_t st = check_w4_desc(&d->w);
    if (st != MOM_OK) return st;
    if (d->w.count != 1) return MOM_ERR_INVALID_ARG;
    const int bytes = element_bytes(d->x_dtype);
    if (!bytes || !is_float_type(d->y_dtype)) return MOM_ERR_DTYPE;
    const bool eight = bytes == 1;
    if (!is_group(d->x_group) || (!eight && d->x_group != 0)) return MOM_ERR_INVALID_ARG;
    if (d->tokens > (1 << 20)) return MOM_ERR_LIMIT;
    if ((d->x_stride != 0 && d->x_stride < d->w.cols) || (d->y_stride != 0 && d->y_stride < d->w.rows) ||
        (d->add_stride > 0 && d->add_stride < d->w.rows) || d->add_stride < -1)
        return MOM_ERR_INVALID_ARG;
    if (d->tokens == 0) return MOM_OK;
    if (!container || !x || !y || eight != (x_scales != nullptr)) return MOM_ERR_INVALID_ARG;
    const int y_bytes = element_bytes(d->y_dtype);
    if (!aligned_to(container, WS_ALIGN) || !aligned_to(x, bytes) || !aligned_to(x_scales, 4) || !aligned_to(add, y_bytes) || !aligned_to(y, y_bytes))
        return MOM_ERR_ALIGNMENT;
    int sm_count = 0;
    st = (mom_status_t)current_sm100(nullptr, &sm_count);
    if (st != MOM_OK) return st;

    W4ProductArgs a;
    a.w = w4_view(d->w, container);
    a.x = x; a.add = add; a.x_scales = x_scales; a.y = y;
    a.x_stride = d->x_stride ? d->x_stride : d->w.cols;
    a.y_stride = d->y_stride ? d->y_stride : d->w.rows;
    a.add_stride = d->add_stride == -1 ? 0 : d->add_stride ? d->add_stride : d->w.rows;
    a.tokens = (int)d->tokens;
    a.y_dtype = d->y_dtype;
    a.x_groups = eight ? (int)groups_of(d->w.cols, d->x_group) : 1;
    a.x_group_shift = group_shift(d->x_group);
    a.wide = aligned_to(x, 16) && (a.x_stride * bytes) % 16 == 0;
    const int per = stretches_per_scale(d->w.group, d->x_group);
    // Up to eight tokens are one column block of mma.sync, which needs no tensor memory and no operand tile of 128 rows; beyond, every
    // eight tokens would cost as many MMAs and reads of x again (16 tokens on mma.sync / tcgen05, us: 8192 x 8192 in bf16 23.7 / 20.8, in
    // e4m3 24.6 / 24.2, 28672 x 8192 81 / 64, 14336 x 4096 in f32 50 / 24.5; the other way round only in small ones, 1024 x 1024 6.2 / 6.7).
    const cudaError_t e = (a.tokens > 8 ? launch_w4_product_tc : launch_w4_product)(a, d->x_dtype, per, sm_count, stream);
    return e == cudaSuccess ? MOM_OK : MOM_ERR_CUDA;
}
