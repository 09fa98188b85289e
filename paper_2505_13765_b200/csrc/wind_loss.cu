// Losses of the output layer z = W x + b over many rows x, without keeping the logits (sm_100a):
//
//     labels    loss_r = lse_v(z_rv) - z_r,t(r)
//     distill   loss_r = tau^2 sum_k q_rk (ln q_rk - ln p_r,i(r,k)),  q_r = softmax_k(y_rk / tau),  p_r = softmax_v(z_rv / tau)
//     gradient  g_rv = s_r (p_rv - [sum of q_rk with i(r,k) = v]),  dx = g W,  dW = g^T x,  db = sum_r g_r
//               (labels: q is one entry of weight 1, tau = 1; s_r is the loss's weight, times tau)
//
// Both losses are one computation: a softmax over all outputs against a target distribution of K >= 1 entries.
//
//     loss_list     the teacher's entries of a row to probabilities, sorted by label
//     loss_gather   rows that count, one behind the other, as tensor-core operands: padding costs nothing from here on; W as a
//                   tensor-core operand, where it is not one already
//     loss_gemm     FORWARD   tiles of logits on the tensor cores; of each tile's row only (maximum, sum of exponentials, sum of q z)
//                             leave the chip
//                   LOGITS    the same tiles again, turned into g, for a piece of the outputs
//                   PRODUCTS  dx += g W and dW = g^T x of that piece, g as both operands' layouts need it: rows are contiguous along
//                             the outputs, which is K of the first product and M of the second (the matrix descriptors take either)
//     loss_combine  a row's partial results to its loss and log-sum-exp
//     loss_finish   partial sums of dx / dW, where a product is cut along its K to fill the chip; db
//
// Tiles: 128 x 256 of bf16 (narrower where that fills the chip better), 256 x 256 by two CTAs for wide rows and many tiles, 128 x 128
// of fp32 and of up to 256 rows.  g in pieces of the outputs and the logits made twice: keeping all of g, or the logits between the two
// calls, would take 2 N n_out bytes, and making logits again costs a quarter of a step's products.
//
// fp32 operands are cut into three bf16 parts, x = x1 + x2 + x3 with 8 bits each, and a product into the six of nine part products
// that are not below 2^-24 of it: x1 w1 + (x1 w2 + x2 w1) + (x1 w3 + x2 w2 + x3 w1), smallest first, in one fp32 accumulator per K
// block.  That is fp32 arithmetic at a sixth of the bf16 rate: 1999 rows, H = 640, 1025 outputs go through their four products at 104
// TFLOP/s of fp32 over the whole step, launches, parts and sums included (the fp32 units' nominal peak is 74.5).
//
// Rounding: logits, exponentials, sums and db stay in fp32.  g is rounded to bf16 (two parts of it up to 256 rows, three for fp32
// models) because it is a tensor-core operand; dx and dW are accumulated in fp32 and rounded once.
//
// What bounds it, loss and gradient together (B200; floor: 8 N H n_out operations at a large matrix product's 1625 TFLOP/s):
//     4096 rows, H = 2048, 65536 outputs     3.45 ms, floor 2.7: the tensor cores under the power limit (3.2 at the rate that a matrix product
//                                            keeps up for seconds), and in the logits eight epilogue warps that hold sums in registers
//     8003 rows, H = 1024, 8193 outputs      455 to 465 us, floor 298: the same, the epilogue of LOGITS, and last waves of equal tiles
//     20011 rows (35 % padding), 640, 1025   112 us, floor 42: FORWARD 21, LOGITS 26 (6700 cycles of epilogue a tile, waits for tensor
//                                            memory and between warps, against 5200 of products), PRODUCTS 38, gathering 2 x 11.5 at
//                                            2.9 TB/s, joining and sums 11
//     1 row, 1024, 8193 (loss)               12 us, floor 2.6: a chain of two kernels (11.3 in a graph of ten), W read at 5 TB/s
//
// Every wait on an mbarrier is bounded: after about two seconds the CTA marks the workspace as timed out, frees its tensor memory and returns.
#include <cuda.h>
#include <cudaTypedefs.h>
#include <math_constants.h>

#include <algorithm>
#include <atomic>
#include <cstddef>
#include <mutex>

#include "wind_internal.cuh"
#include "wind_loop.cuh"
#include "wind_loop_cl.cuh"   // cl_rank, cl_map, cl_barrier
#include "wind_loss.cuh"
#include "wind_ptx.cuh"

namespace wind {

// ---------------------------------------------------------------------------
// sizes
// ---------------------------------------------------------------------------
constexpr int LT_BAND = 16;               // row tiles that are worked on together (see unit_of)
constexpr int ROWS_COUNTED = 32768;       // longer calls have the rows that count counted by a kernel of its own, so many at a time
constexpr int PANEL_BYTES = 64 * BK * 2;  // 64 x 64 bf16
constexpr int kFillCtas = 148;            // CTAs that a product is cut for
constexpr int kNarrowTiles = 4 * kFillCtas;   // so many tiles or more are not made narrower, nor their sums cut to fill the chip
constexpr int kSumAdditions = 4096;       // of an accumulator of dx and dW: at most 4096 x 2^-23 = 2^-11 is lost, of results rounded to 2^-8

static inline int up(long long a, int b) { return (int)((a + b - 1) / b * b); }
static inline int cdiv(long long a, int b) { return (int)((a + b - 1) / b); }

// ---------------------------------------------------------------------------
// rows: which count, and their operands
// ---------------------------------------------------------------------------
enum Mark : uint8_t { ROW_NONE = 0, ROW_COUNTS = 1, ROW_BAD = 2 };   // BAD: a label outside [-1, n_out)

struct RowsParams {
    LossCtrl* ctrl;
    int N, n_out, K, H, Hp, Npad, x_vec, dx_vec, grad;
    int32_t* next; int n_next; // units taken by the products' kernels
    int row_blocks;            // blocks of loss_gather that take rows; those behind them lay W out
    const void* w; int64_t ldw; int w_vec; __nv_bfloat16* wc;
    float* db;                 // where its only writers are the tiles of logits
    const void* dw;
    int counted;               // counts[] holds the rows that count, of every ROWS_COUNTED rows
    int per_block;             // rows of a block of loss_gather, a multiple of 8
    float tau;
    const int32_t* target; const int32_t* ids; const float* y;
    const void* x; int64_t ldx;
    int32_t* counts; uint8_t* mark; int32_t* src; int32_t* target_c; float* scale_c; float* nlse_c; int2* list; uint8_t* where; int where_ld; float* ent;
    __nv_bfloat16* xc;
    float* loss; float* lse_out;
    const float* lse; const float* dloss;
    void* dx; int64_t lddx;
};

__device__ __forceinline__ uint8_t mark_of(const int32_t* target, const uint8_t* mark, int n_out, int r) {
    if (mark) return mark[r];
    const int t = target[r];
    return t == -1 ? ROW_NONE : (t >= 0 && t < n_out ? ROW_COUNTS : ROW_BAD);
}

__device__ __forceinline__ uint8_t row_mark(const RowsParams& p, int r) { return mark_of(p.target, p.K ? p.mark : nullptr, p.n_out, r); }

constexpr int WHERE_WORDS = 512;
constexpr uint32_t NO_LABEL = 0xffffffu;   // (n_out is below 2^24)

// The teacher's list of a row, a warp each: probabilities over the entries that are there, and the entries by rising label (equal
// labels in their order), so that the epilogues walk a list along their columns: the keys label * 256 + entry, PER to a lane, go through
// a bitonic network of exchanges between lanes.  (Finding a key's place by counting the keys below it is K^2 / 32 comparisons a lane:
// 38 us instead of 23 for 19677 lists of 74, 36 instead of 14 for 9924 of 115, 7.0 instead of 5.9 for 6007 of 16.)  `where` has for every
// 32nd output the number of entries below it (255 for 256), a byte each: the epilogues start there (searching, 16 warps a tile, cost
// them 4000 cycles a tile).
template <int PER>
__global__ void __launch_bounds__(256) loss_list_kernel(const RowsParams p) {
    __shared__ __align__(16) uint32_t s_where[8][WHERE_WORDS];
    __shared__ float s_q[8][32 * PER];
    let_next_start();
    wait_for_previous();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int r = blockIdx.x * 8 + warp;
    if (r >= p.N) return;
    const int32_t* ids = p.ids + (size_t)r * p.K;
    const float* y = p.y + (size_t)r * p.K;
    uint32_t key[PER];
    float v[PER];
    int id[PER];
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        const int k = lane + 32 * i;
        id[i] = k < p.K ? ids[k] : -1;
        v[i] = k < p.K ? y[k] : 0.f;
    }
    float top = -CUDART_INF_F;
    int flags = 0;   // 1: an entry outside the outputs, 2: NaN
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        const bool there = id[i] >= 0 && id[i] < p.n_out;
        if (id[i] < -1 || id[i] >= p.n_out) flags |= 1;
        if (there && v[i] != v[i]) flags |= 2;
        if (there) top = fmaxf(top, v[i]);
        else v[i] = -CUDART_INF_F;
        key[i] = lane + 32 * i < p.K ? (there ? (uint32_t)id[i] : NO_LABEL) << 8 | (uint32_t)(lane + 32 * i) : 0xffffffffu;   // (behind the list: below no key)
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
    flags = __reduce_or_sync(0xffffffffu, flags);
    float sum = 0.f, e[PER];
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        const bool some = v[i] != -CUDART_INF_F;
        v[i] = some ? (v[i] - top) / p.tau : 0.f;
        e[i] = some ? expf(v[i]) : 0.f;
        sum += e[i];
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
    const float log_sum = logf(sum);
    float ent = 0.f;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        const float q = e[i] != 0.f ? e[i] / sum : 0.f;
        if (q != 0.f) ent += q * (v[i] - log_sum);
        s_q[warp][lane + 32 * i] = q;
    }
    // position of a key in the network: lane * PER + i
#pragma unroll
    for (int size = 2; size <= 32 * PER; size *= 2) {
#pragma unroll
        for (int stride = size / 2; stride > 0; stride /= 2) {
            if (stride >= PER) {
                const bool low = ((lane & (stride / PER)) == 0) == ((lane * PER & size) == 0);
#pragma unroll
                for (int i = 0; i < PER; ++i) {
                    const uint32_t other = __shfl_xor_sync(0xffffffffu, key[i], stride / PER);
                    key[i] = low ? min(key[i], other) : max(key[i], other);
                }
            } else {
#pragma unroll
                for (int i = 0; i < PER; ++i) {
                    if (i & stride) continue;
                    const bool rising = ((lane * PER + i) & size) == 0;
                    const uint32_t a = key[i], b = key[i + stride];
                    key[i] = rising ? min(a, b) : max(a, b);
                    key[i + stride] = rising ? max(a, b) : min(a, b);
                }
            }
        }
    }
    __syncwarp();
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        const int at = lane * PER + i;
        const int label = key[i] >> 8 == NO_LABEL ? 0x7fffffff : (int)(key[i] >> 8);
        if (at < p.K) p.list[(size_t)r * p.K + at] = make_int2(label, __float_as_int(s_q[warp][key[i] & 255]));
        if (at == 255) key[i] = 0xffffffffu;       // (never the reason to start behind entry 255)
    }
    // `where`: how many labels lie in each 32 outputs, a byte each, and their running sums
    uint32_t* w = s_where[warp];
    uint32_t below = 0;
    for (int b0 = 0; b0 < p.where_ld; b0 += 4 * WHERE_WORDS) {
        const int words = min(WHERE_WORDS, (p.where_ld - b0) / 4);
        __syncwarp();
        for (int i = lane; i < words; i += 32) w[i] = 0;
        __syncwarp();
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            const int at = (int)(key[i] >> 13) + 1 - b0;      // label / 32 + 1
            if (key[i] >> 8 != NO_LABEL && at >= 0 && at < 4 * words) atomicAdd(&w[at >> 2], 1u << (8 * (at & 3)));
        }
        __syncwarp();
        for (int i0 = 0; i0 < words; i0 += 32) {
            uint32_t sums = i0 + lane < words ? w[i0 + lane] * 0x01010101u : 0u;      // running sums of the word's bytes
            uint32_t upto = sums >> 24;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const uint32_t v = __shfl_up_sync(0xffffffffu, upto, o);
                if (lane >= o) upto += v;
            }
            sums += (below + upto - (sums >> 24)) * 0x01010101u;
            if (i0 + lane < words) reinterpret_cast<uint32_t*>(p.where + (size_t)r * p.where_ld + b0)[i0 + lane] = sums;
            below += __shfl_sync(0xffffffffu, upto, 31);
        }
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) ent += __shfl_xor_sync(0xffffffffu, ent, o);
    if (lane == 0) {
        p.mark[r] = (flags & 1) ? ROW_BAD : ((flags & 2) || top != -CUDART_INF_F ? ROW_COUNTS : ROW_NONE);
        p.ent[r] = ent;
    }
}

constexpr int COUNTED_BAD = 1 << 30;   // a row among them is none

// Rows that count, of every ROWS_COUNTED rows: only for calls so long that the blocks of loss_gather should not count them all.
__global__ void __launch_bounds__(256) loss_count_kernel(const RowsParams p) {
    __shared__ int s_count;
    let_next_start();
    wait_for_previous();
    if (threadIdx.x == 0) s_count = 0;
    __syncthreads();
    int n = 0, bad = 0;
#pragma unroll 8
    for (int i = threadIdx.x; i < ROWS_COUNTED; i += 256) {
        const int r = blockIdx.x * ROWS_COUNTED + i;
        const uint8_t m = r < p.N ? row_mark(p, r) : (uint8_t)ROW_NONE;
        n += m == ROW_COUNTS;
        bad |= m == ROW_BAD;
    }
    atomicAdd(&s_count, n);
    if (bad) atomicOr(&s_count, COUNTED_BAD);
    __syncthreads();
    if (threadIdx.x == 0) p.counts[blockIdx.x] = s_count;
}

// Eight columns of a row as fp32; columns from H on are zero.
template <bool F32>
__device__ __forceinline__ void load8(const void* row, int c, int H, bool vec, float* v) {
    if (vec && c + 8 <= H) {
        if (F32) {
            const float4* s = reinterpret_cast<const float4*>(static_cast<const float*>(row) + c);
            const float4 a = s[0], b = s[1];
            v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w; v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
        } else {
            const uint4 a = *reinterpret_cast<const uint4*>(static_cast<const __nv_bfloat16*>(row) + c);
            const uint32_t w[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
            for (int i = 0; i < 4; ++i) { v[2 * i] = __uint_as_float(w[i] << 16); v[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u); }
        }
        return;
    }
#pragma unroll
    for (int i = 0; i < 8; ++i)
        v[i] = c + i < H ? (F32 ? static_cast<const float*>(row)[c + i] : __bfloat162float(static_cast<const __nv_bfloat16*>(row)[c + i])) : 0.f;
}

// x = p1 + p2 + p3 with eight bits each (nearest; downwards where nearest would overflow).  Infinities and NaN stand in p1 alone.
__device__ __forceinline__ void split3(float x, float* part) {
    float a = __bfloat162float(__float2bfloat16_rn(x));
    if (isinf(a) && !isinf(x)) a = __uint_as_float(__float_as_uint(x) & 0xffff0000u);
    const float r = isfinite(a) ? x - a : 0.f;
    const float b = __bfloat162float(__float2bfloat16_rn(r));
    part[0] = a; part[1] = b; part[2] = r - b;
}

template <bool F32>
__device__ __forceinline__ void store8(__nv_bfloat16* dst, size_t plane, const float* v) {
    if constexpr (!F32) {
        *reinterpret_cast<uint4*>(dst) = make_uint4(pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]), pack_bf16x2(v[4], v[5]), pack_bf16x2(v[6], v[7]));
    } else {
        float s[8][3];
#pragma unroll
        for (int i = 0; i < 8; ++i) split3(v[i], s[i]);
#pragma unroll
        for (int t = 0; t < 3; ++t)
            *reinterpret_cast<uint4*>(dst + t * plane) = make_uint4(pack_bf16x2(s[0][t], s[1][t]), pack_bf16x2(s[2][t], s[3][t]),
                                                                    pack_bf16x2(s[4][t], s[5][t]), pack_bf16x2(s[6][t], s[7][t]));
    }
}

// 256-bit store: a whole sector per thread (16-byte stores from 32 threads to 32 rows send every byte to L2 twice)
__device__ __forceinline__ void store_sector(void* p, const uint32_t* w) {
    asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(p), "r"(w[0]), "r"(w[1]), "r"(w[2]), "r"(w[3]),
                 "r"(w[4]), "r"(w[5]), "r"(w[6]), "r"(w[7])
                 : "memory");
}

// Sixteen neighbouring values in one to three bf16 parts, 32-byte aligned.
template <int PARTS>
__device__ __forceinline__ void store16(__nv_bfloat16* dst, size_t plane, const float* v) {
    uint32_t w[PARTS][8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        if constexpr (PARTS == 1) w[0][i] = pack_bf16x2(v[2 * i], v[2 * i + 1]);
        else {
            float a[3], b[3];
            split3(v[2 * i], a);
            split3(v[2 * i + 1], b);
#pragma unroll
            for (int t = 0; t < PARTS; ++t) w[t][i] = pack_bf16x2(a[t], b[t]);
        }
    }
#pragma unroll
    for (int t = 0; t < PARTS; ++t) store_sector(dst + t * plane, w[t]);
}

template <bool F32>
__device__ __forceinline__ void store_one(void* row, int c, float v) {
    if (F32) static_cast<float*>(row)[c] = v;
    else static_cast<__nv_bfloat16*>(row)[c] = __float2bfloat16_rn(v);
}

// W as tensor-core operands, by `blocks` blocks.
template <bool F32>
__device__ __forceinline__ void pack_w(const RowsParams& p, int block, int blocks) {
    const size_t plane = (size_t)p.n_out * p.Hp;
    const int per_row = p.Hp / 8;
    const long long all = (long long)p.n_out * per_row;
#pragma unroll 2
    for (long long i = (long long)block * 256 + threadIdx.x; i < all; i += (long long)blocks * 256) {
        const int r = (int)(i / per_row), c = (int)(i - (long long)r * per_row) * 8;
        float v[8];
        load8<F32>(static_cast<const uint8_t*>(p.w) + (size_t)r * p.ldw * (F32 ? 4 : 2), c, p.H, p.w_vec, v);
        store8<F32>(p.wc + (size_t)r * p.Hp + c, plane, v);
    }
}

// A block takes per_block rows.  Where its first row that counts goes is the number of such rows before it, which every block finds out
// for itself: reading up to ROWS_COUNTED marks from L2 is quicker than another launch.
template <bool F32>
__global__ void __launch_bounds__(256) loss_gather_kernel(const RowsParams p) {
    __shared__ int s_before[8];
    __shared__ uint32_t s_ballot[8];
    __shared__ uint8_t s_mark[256], s_row[256];
    let_next_start();
    wait_for_previous();
    if ((int)blockIdx.x >= p.row_blocks) {
        pack_w<F32>(p, blockIdx.x - p.row_blocks, gridDim.x - p.row_blocks);
        return;
    }
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int r0 = blockIdx.x * p.per_block, r1 = min(r0 + p.per_block, p.N);
    int before = 0, first = 0;
    bool bad = false;
    if (p.counted) {
        first = r0 / ROWS_COUNTED;
        for (int i = threadIdx.x; i < first; i += 256) {
            before += p.counts[i] & (COUNTED_BAD - 1);
            bad |= (p.counts[i] & COUNTED_BAD) != 0;
        }
        first *= ROWS_COUNTED;
    }
    // (first and r0 are multiples of 8)
    if (p.K) {
        for (int r = first + 8 * (int)threadIdx.x; r < r0; r += 8 * 4 * 256) {
            uint2 m[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) m[i] = r + i * 2048 < r0 ? *reinterpret_cast<const uint2*>(p.mark + r + i * 2048) : make_uint2(0, 0);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                before += __popc(m[i].x & 0x01010101u) + __popc(m[i].y & 0x01010101u);
                bad |= ((m[i].x | m[i].y) & 0x02020202u) != 0;
            }
        }
    } else {
        const bool vec = reinterpret_cast<uintptr_t>(p.target) % 16 == 0;
        for (int r = first + 4 * (int)threadIdx.x; r < r0; r += 4 * 8 * 256) {
            int t[8][4];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const int at = r + i * 1024;
                if (at >= r0) { t[i][0] = t[i][1] = t[i][2] = t[i][3] = -1; }
                else if (vec) {
                    const int4 q = *reinterpret_cast<const int4*>(p.target + at);
                    t[i][0] = q.x; t[i][1] = q.y; t[i][2] = q.z; t[i][3] = q.w;
                } else {
#pragma unroll
                    for (int k = 0; k < 4; ++k) t[i][k] = p.target[at + k];
                }
            }
#pragma unroll
            for (int i = 0; i < 32; ++i) {
                const int v = t[i / 4][i % 4];
                before += v >= 0 && v < p.n_out;
                bad |= v < -1 || v >= p.n_out;
            }
        }
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) before += __shfl_xor_sync(0xffffffffu, before, o);
    const uint8_t mine = r0 + (int)threadIdx.x < r1 ? row_mark(p, r0 + threadIdx.x) : (uint8_t)ROW_NONE;
    const uint32_t ballot = __ballot_sync(0xffffffffu, mine == ROW_COUNTS);
    if (lane == 0) { s_before[warp] = before; s_ballot[warp] = ballot; }
    s_mark[threadIdx.x] = mine;
    bad = __syncthreads_or(bad || mine == ROW_BAD);
    // s_row: the block's rows that count, in order, and behind them, from the end, the others
    int mine_before = __popc(ballot & ((1u << lane) - 1u)), here = 0, first_pos = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        first_pos += s_before[i];
        here += __popc(s_ballot[i]);
        if (i < warp) mine_before += __popc(s_ballot[i]);
    }
    const int rows = r1 - r0, me = (int)threadIdx.x;
    if (me < rows) {
        if (mine == ROW_COUNTS) s_row[mine_before] = (uint8_t)me;
        else s_row[rows - 1 - (me - mine_before)] = (uint8_t)me;
    }
    __syncthreads();
    const size_t plane = (size_t)p.Npad * p.Hp;
    const size_t es = F32 ? 4 : 2;
    // eight columns a thread, over all rows of the block; four loads of a thread are under way together
    const int per_row = p.Hp / 8, chunks = here * per_row;
    if (!F32 && p.x_vec) {
        const uint4* x = static_cast<const uint4*>(p.x);
        uint4* out = reinterpret_cast<uint4*>(p.xc);
        const int64_t ld = p.ldx / 8;
        const int in_row = p.H / 8;
        for (int i0 = me; i0 < chunks; i0 += 4 * 256) {
            uint4 v[4];
            int to[4];
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const int i = i0 + q * 256, k = i / per_row, c = i - k * per_row;
                to[q] = k * per_row + c;
                v[q] = i < chunks && c < in_row ? x[(size_t)(r0 + s_row[k]) * ld + c] : make_uint4(0, 0, 0, 0);
            }
#pragma unroll
            for (int q = 0; q < 4; ++q)
                if (i0 + q * 256 < chunks) out[(size_t)first_pos * per_row + to[q]] = v[q];
        }
    } else {
#pragma unroll 2
        for (int i = me; i < chunks; i += 256) {
            const int k = i / per_row, c = (i - k * per_row) * 8;
            float v[8];
            load8<F32>(static_cast<const uint8_t*>(p.x) + (size_t)(r0 + s_row[k]) * p.ldx * es, c, p.H, p.x_vec, v);
            store8<F32>(p.xc + (size_t)(first_pos + k) * p.Hp + c, plane, v);
        }
    }
    if (me < here) {
        const int r = r0 + s_row[me], j = first_pos + me;
        p.src[j] = r;
        if (p.K == 0) p.target_c[j] = p.target[r];
        if (p.grad) {
            p.scale_c[j] = (p.dloss ? p.dloss[r] : 1.f) * p.tau;
            p.nlse_c[j] = p.lse[r];
        }
    }
    if (!p.grad) {
        if (me >= here && me < rows) {
            const int r = s_row[me];
            const float fill = s_mark[r] == ROW_BAD ? CUDART_NAN_F : 0.f;
            p.loss[r0 + r] = fill;
            p.lse_out[r0 + r] = fill;
        }
    } else if (p.dx) {
        for (int k = here + warp; k < rows; k += 8) {
            const int r = s_row[k];
            const float fill = s_mark[r] == ROW_BAD ? CUDART_NAN_F : 0.f;
            uint8_t* row = static_cast<uint8_t*>(p.dx) + (size_t)(r0 + r) * p.lddx * es;
            if (p.dx_vec) {
                const uint32_t w = F32 ? __float_as_uint(fill) : pack_bf16x2(fill, fill);
                for (int c = lane; c < p.H * (int)es / 16; c += 32) reinterpret_cast<uint4*>(row)[c] = make_uint4(w, w, w, w);
            } else {
                for (int c = lane; c < p.H; c += 32) store_one<F32>(row, c, fill);
            }
        }
    }
    if ((int)blockIdx.x == p.row_blocks - 1) {
        const int total = first_pos + here;
        // dW sums over K blocks of 64 rows: zeros behind the last one.  (Other products only make rows of it that nobody looks at.)
        if (threadIdx.x == 0) {   // (this block has seen every mark)
            p.ctrl->status = bad ? WIND_ERR_INVALID_ARG : WIND_OK;
            p.ctrl->n_rows = total;
        }
        for (int i = threadIdx.x; i < p.n_next; i += 256) p.next[i] = 0;
        const float zero[8] = {};
        if (p.dw)
            for (int j = total + warp; j < (total + 63) / 64 * 64; j += 8)
                for (int c = lane * 8; c < p.Hp; c += 256) store8<F32>(p.xc + (size_t)j * p.Hp + c, plane, zero);
        if (p.db && total == 0)      // (no tile of logits is there to write it)
            for (int v = threadIdx.x; v < p.n_out; v += 256) p.db[v] = 0.f;
    }
}

// ---------------------------------------------------------------------------
// The products: a persistent tcgen05 GEMM with three epilogues
// ---------------------------------------------------------------------------
enum LossMode { FORWARD = 0, LOGITS = 1, PRODUCTS = 2 };
// Operands, by the parts of g: bf16; bf16 with g in two parts, for calls of few rows; fp32 (three parts of every operand).
// Few rows: an error that many rows' sums and norms average out stands alone in one, and the products' time is that of reading W and
// writing dW, whatever the parts.  (With one part dx and dW of three rows were 0.0029 off, 0.0017 being bf16's own rounding.)
// BF16_LONG: BF16 for logits of more than kLongBlocks K blocks; its products and its one part of g are BF16's.
enum LossKind { BF16 = 1, BF16_FINE = 2, F32 = 3, BF16_LONG = 4 };
__host__ __device__ constexpr int parts_of_g(int kind) { return kind == BF16_LONG ? 1 : kind; }
constexpr int kFineRows = 256;
constexpr int kLongBlocks = 16;   // K blocks that an accumulator of bf16 logits takes: 64 additions

struct LossGemm {
    LossCtrl* ctrl;
    int n_out, H, Hp, Npad, K;
    int kb;                       // K blocks of the logits
    int tn;                       // columns of a tile: 64, 128 or 256
    int stages, stage_bytes;      // the ring of K blocks (see ring_of)
    int a_rows;                   // rows that a fetch of x, or of g for dx, brings; b_bytes: what lies between the parts of B
    int b_bytes;
    int w_panels;                 // PRODUCTS: W's columns are whole groups of 64 (map_b as panel_map makes it)
    int v0, cols, n_vt;           // this piece's first output, its outputs (to n_out at most) and tiles
    int32_t* next;                // units that were taken, beyond the CTAs' first ones; null: CTAs take them in turn
    int direct;                   // FORWARD: x as the caller has it, this many rows; 0: gathered rows
    int stall;                    // test hook: the first CTA's or pair's wait that cannot end (1: operands, 2: products, 3: the next unit)
    float rtau;                   // 1 / tau
    const float* bias;
    const int32_t* src; const int32_t* target; const int2* list; const uint8_t* where; int where_ld;
    float *pm, *ps, *pq;          // FORWARD: [parts][Npad]; where a row has one part its results instead:
    float *loss, *lse; const float* ent; float tau;
    const float* scale; const float* nlse;
    __nv_bfloat16* g; int ldg; size_t g_plane; float* dbp;   // LOGITS
    // PRODUCTS
    int dx_first;                 // whether dx's units are the longer ones
    int ht, s_dx, s_dw, add_dx;   // tiles of H, parts of the sums, whether dx's partial sums are added to
    float *sdx, *sdw; int slab_rows_dw;   // partial sums, or null: straight to dx / dw
    void* dx; int64_t lddx; int dx_vec; int want_dx;         // vec: what rows are aligned to, 0: nothing, 1: 16 bytes, 2: 32 bytes
    void* dw; int64_t lddw; int dw_vec; int want_dw;
};

// Shape of a kernel.  A stage holds a K block of every part of both operands, and all part products are made from it: fp32 fetches 96 KB
// for six products of 128 x 128 x 64 (64 bytes of L2 a cycle and SM; a fetch for each product would be 128).
template <int MODE, int KIND>
struct Shape {
    // Tensor cores cut where they add; over a long K that is up to 2^-23 an addition, all one way (a single row of H = 1024 had a loss
    // 3e-6 off).  Logits of fp32 models and of calls of few rows: an accumulator takes one K block, whose sum is added up in registers;
    // logits of long bf16 rows: sixteen of them, which takes FORWARD of 4096 x 2048 x 65536 from 648 to 673 us, LOGITS from 700 to 755 (eight
    // epilogue warps have room for the sums, sixteen do not); with eight K blocks an accumulator 717 and 852.
    static constexpr bool SUMS = KIND == F32 || ((KIND == BF16_FINE || KIND == BF16_LONG) && MODE != PRODUCTS);
    static constexpr int ACC_BLOCKS = SUMS ? (KIND == BF16_LONG ? kLongBlocks : 1) : 1 << 30;   // K blocks that an accumulator takes
    static constexpr int TN = SUMS && KIND != BF16_LONG ? 128 : 256;                         // most columns of a tile (BM = 128 rows)
    static constexpr int A_PARTS = KIND == F32 ? 3 : (KIND == BF16_FINE && MODE == PRODUCTS ? 2 : 1), B_PARTS = KIND == F32 ? 3 : 1;
    static constexpr int TERMS = KIND == F32 ? 6 : A_PARTS;
    // Groups of four epilogue warps (one per tensor-memory lane quadrant), each with its columns of a tile.  A row of logits is a chain
    // of maxima, exponentials and sums: 16 warps hide more of it than 8 (which is what sums in registers leave room for).
    static constexpr int GROUPS = MODE != PRODUCTS && !SUMS ? 4 : 2;
    static constexpr int EPI = 128 * GROUPS, THREADS = 64 + EPI, CHUNKS = TN / GROUPS / 32;
    // Part products, smallest first: the parts of A and B of each (fp32: 20 02 11 10 01 00; fine: 10 00).
    static __device__ __forceinline__ constexpr int a_part(int t) { return KIND == F32 ? (0x001102 >> (4 * t)) & 3 : TERMS - 1 - t; }
    static __device__ __forceinline__ constexpr int b_part(int t) { return KIND == F32 ? (0x010120 >> (4 * t)) & 3 : 0; }
};
constexpr int kRingBytes = 196608 + A_STAGE_BYTES;   // 4 full stages of bf16, 3 of fine, 2 of fp32, and what a short A reads behind its last
constexpr int kMaxStages = 16;
__host__ __device__ constexpr int group_cols(int tn, int groups) { return tn / groups > 32 ? tn / groups : 32; }

// K-major tiles as in smem_desc_sw128.  MN-major ones: panels of 64 (M or N) x 64 (K) bf16, a K row of a panel being 128 bytes: 8 K rows
// are a swizzle atom of 1024 bytes (stride byte offset), panels stand PANEL_BYTES apart (leading byte offset).
__device__ __forceinline__ uint64_t smem_desc_mn(uint32_t smem_addr) {
    uint64_t d = 0;
    d |= (uint64_t)((smem_addr & 0x3FFFFu) >> 4);
    d |= (uint64_t)(PANEL_BYTES >> 4) << 16;
    d |= (uint64_t)(1024 >> 4) << 32;
    d |= (uint64_t)1 << 46;
    d |= (uint64_t)2 << 61;
    return d;
}

// The instruction wants the whole warp at once, and a vote does not bring lanes together that took different ways before, as they do
// out of a long wait on an mbarrier: they meet here.
__device__ __forceinline__ void tmem_ld32(uint32_t taddr, float* v) {
    uint32_t r[32];
    __syncwarp();
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,%23,"
        "%24,%25,%26,%27,%28,%29,%30,%31}, [%32];"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]),
          "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]), "=r"(r[17]), "=r"(r[18]),
          "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]), "=r"(r[25]), "=r"(r[26]), "=r"(r[27]),
          "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
        : "r"(taddr)
        : "memory");
    asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
#pragma unroll
    for (int i = 0; i < 32; ++i) v[i] = __uint_as_float(r[i]);
}

__device__ __forceinline__ float exp2_fast(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
constexpr float kLog2e = 1.4426950408889634f;

// v[at], by halves: 31 selections and five comparisons (a comparison and a selection for each value: FORWARD of 6007 rows with 16
// entries 15.2 us instead of 14.6)
__device__ __forceinline__ float pick32(const float* v, int at) {
    float t[16];
#pragma unroll
    for (int i = 0; i < 16; ++i) t[i] = (at & 16) ? v[i + 16] : v[i];
#pragma unroll
    for (int h = 8; h > 0; h >>= 1)
#pragma unroll
        for (int i = 0; i < h; ++i) t[i] = (at & h) ? t[i + h] : t[i];
    return t[0];
}

// What a CTA's roles need to know about a piece of work.
struct __align__(8) Unit {
    int mt, nt;          // row tile of A, column tile of B; mt -1: there is none
    int k0, nk;          // K blocks
    int dw;              // PRODUCTS: dW (else dx)
    int part;            // PRODUCTS: which part of the sum
};

template <int MODE, int TM>
__device__ __forceinline__ uint32_t count_units(const LossGemm& p, int n_rows) {
    const int mtc = (n_rows + TM - 1) / TM;
    if (MODE != PRODUCTS) return (uint32_t)mtc * p.n_vt;
    uint32_t n = 0;
    if (p.want_dx) n += (uint32_t)p.s_dx * mtc * p.ht;
    if (p.want_dw) n += (uint32_t)p.s_dw * ((p.cols + TM - 1) / TM) * p.ht;
    return n;
}

// (There are below 2^31 units: the entry points see to that.)  Tiles of TM rows.  Logits: bands of LT_BAND x 128 rows, in a band row tile fastest, so that the CTAs at work share few tiles of x and of W; last tiles of
// at most half the columns (1024 labels and the blank) come behind all others.  Products: the longer ones first.  CTAs take the next
// unit when they are through with one, and what is short at the end fills the gaps.
template <int MODE, int TM>
__device__ __forceinline__ Unit unit_of(const LossGemm& p, int n_rows, uint32_t u, uint32_t n_units) {
    Unit t{};
    if (u >= n_units) {
        t.mt = -1;
        return t;
    }
    constexpr int BAND = LT_BAND * BM / TM;
    const int mtc = (n_rows + TM - 1) / TM;
    if (MODE != PRODUCTS) {
        const int rest = p.cols - (p.n_vt - 1) * p.tn, wide = p.n_vt - (p.n_vt > 1 && 2 * rest <= p.tn);
        t.nk = p.kb;
        const uint32_t n_wide = (uint32_t)mtc * wide;
        if (u >= n_wide) {
            t.nt = wide;
            t.mt = (int)(u - n_wide);
            return t;
        }
        const uint32_t per_band = (uint32_t)BAND * wide;
        const int band = (int)(u / per_band);
        const int r = (int)(u - band * per_band), in_band = min(BAND, mtc - band * BAND);
        t.nt = in_band == BAND ? r / BAND : r / in_band;
        t.mt = band * BAND + (r - t.nt * in_band);
        return t;
    }
    const uint32_t n_dx = p.want_dx ? (uint32_t)p.s_dx * mtc * p.ht : 0, n_dw = p.want_dw ? (uint32_t)p.s_dw * ((p.cols + TM - 1) / TM) * p.ht : 0;
    t.dw = p.dx_first ? u >= n_dx : u < n_dw;
    if (t.dw == p.dx_first) u -= t.dw ? n_dx : n_dw;
    const int tiles = (t.dw ? (p.cols + TM - 1) / TM : mtc) * p.ht;
    t.part = (int)(u / tiles);
    const int r = (int)(u - (uint32_t)t.part * tiles);
    t.mt = r / p.ht;
    t.nt = r - t.mt * p.ht;
    const int kb = ((t.dw ? n_rows : p.cols) + BK - 1) / BK, s = t.dw ? p.s_dw : p.s_dx;
    if (s > 1) {
        t.k0 = (int)((long long)kb * t.part / s);
        t.nk = (int)((long long)kb * (t.part + 1) / s) - t.k0;
    } else {
        t.nk = kb;
    }
    return t;
}
// A CTA's first unit is that of its number; the others are handed on through a ring, by the one thread that fetches operands and
// takes them, to the one that issues the products and to the epilogue.  They go as tiles, worked out while earlier operands are under
// way: left to the issuing thread, that stood 1200 cycles between one tile's products and the next one's.
constexpr int UNITS = 4;
struct UnitRing {
    uint64_t full[UNITS], empty[UNITS];
    Unit unit[UNITS];
};
__device__ __forceinline__ Unit read_unit(const Unit* at) {
    const volatile long long* w = reinterpret_cast<const volatile long long*>(at);
    long long v[3] = {w[0], w[1], w[2]};
    Unit t;
    memcpy(&t, v, sizeof(t));
    return t;
}
__device__ __forceinline__ void write_unit(Unit* at, const Unit& t) {
    long long v[3];
    memcpy(v, &t, sizeof(t));
    volatile long long* w = reinterpret_cast<volatile long long*>(at);
    w[0] = v[0]; w[1] = v[1]; w[2] = v[2];
}
// ---- two CTAs on neighbouring SMs that make one tile of 256 rows (cta_group::2) ----
// Each fetches its 128 rows of A and half the columns of B; the first one's thread issues the products, which read both shared memories
// and write both tensor memories.  Fetches of both are counted on the first one's barriers.
__device__ __forceinline__ void mbar_arrive_at(uint32_t addr) {   // addr: in any CTA of the cluster
    asm volatile("mbarrier.arrive.release.cluster.shared::cluster.b64 _, [%0];" ::"r"(addr) : "memory");
}
// mbar_wait for a barrier that the other CTA arrives at
__device__ __forceinline__ bool mbar_wait_pair(uint64_t* bar, uint32_t parity, volatile int* abort_flag) {
    unsigned long long t0 = 0;
    for (uint32_t it = 0;; ++it) {
        uint32_t ok;
        asm volatile(
            "{\n\t.reg .pred p;\n\t"
            "mbarrier.try_wait.parity.acquire.cluster.shared::cta.b64 p, [%1], %2, %3;\n\t"
            "selp.u32 %0, 1, 0, p;\n\t}"
            : "=r"(ok)
            : "r"(smem_u32(bar)), "r"(parity), "r"(20000u)
            : "memory");
        if (ok) return true;
        if ((it & 7u) == 7u) {
            if (*abort_flag) return false;
            const unsigned long long now = globaltimer_ns();
            if (t0 == 0) t0 = now;
            else if (now - t0 > kWaitLimitNs) { *abort_flag = 1; return false; }
        }
    }
}
__device__ __forceinline__ void tma_load_3d_pair(void* smem_dst, const CUtensorMap* tmap, int x, int y, int z, uint32_t bar) {   // bar: either CTA's
    asm volatile(
        "cp.async.bulk.tensor.3d.cta_group::2.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];" ::"r"(
            smem_u32(smem_dst)),
        "l"(reinterpret_cast<uint64_t>(tmap)), "r"(x), "r"(y), "r"(z), "r"(bar)
        : "memory");
}
// (4-D: 64 columns, rows, groups of 64 columns, parts: see panel_map)
__device__ __forceinline__ void tma_load_4d(void* smem_dst, const CUtensorMap* tmap, int x, int y, int z, int w, uint64_t* bar) {
    asm volatile(
        "cp.async.bulk.tensor.4d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4, %5}], [%6];" ::"r"(smem_u32(smem_dst)),
        "l"(reinterpret_cast<uint64_t>(tmap)), "r"(x), "r"(y), "r"(z), "r"(w), "r"(smem_u32(bar))
        : "memory");
}
__device__ __forceinline__ void tma_load_4d_pair(void* smem_dst, const CUtensorMap* tmap, int x, int y, int z, int w, uint32_t bar) {
    asm volatile(
        "cp.async.bulk.tensor.4d.cta_group::2.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4, %5}], [%6];" ::"r"(
            smem_u32(smem_dst)),
        "l"(reinterpret_cast<uint64_t>(tmap)), "r"(x), "r"(y), "r"(z), "r"(w), "r"(bar)
        : "memory");
}
__device__ __forceinline__ void tc_mma_bf16_pair(uint32_t tmem_d, uint64_t adesc, uint64_t bdesc, uint32_t idesc, uint32_t accumulate) {
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n\t}" ::"r"(tmem_d),
        "l"(adesc), "l"(bdesc), "r"(idesc), "r"(accumulate)
        : "memory");
}
__device__ __forceinline__ void tc_commit_pair(uint64_t* bar) {    // arrives at that barrier of both CTAs
    asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;" ::"r"(smem_u32(bar)),
                 "h"((uint16_t)3)
                 : "memory");
}
__device__ __forceinline__ void tc_commit_pair_here(uint64_t* bar) {    // arrives at this CTA's alone
    asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(smem_u32(bar)) : "memory");
}
__device__ __forceinline__ void tmem_alloc_pair(uint32_t* slot, uint32_t ncols) {
    asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(slot)), "r"(ncols) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
}
__device__ __forceinline__ void tmem_dealloc_pair(uint32_t taddr, uint32_t ncols) {
    asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(taddr), "r"(ncols) : "memory");
}

// The n-th unit behind the first; mt is -1 where none is left, or the wait ran out.  A pair's first CTA takes the units and leaves each in
// both rings; both tell it when they have read one.
template <bool PAIR>
__device__ __forceinline__ Unit next_unit(UnitRing& ring, uint32_t n, uint32_t rank, volatile int* abort_flag) {
    const uint32_t i = n % UNITS;
    const bool there = PAIR ? mbar_wait_pair(&ring.full[i], (n / UNITS) & 1, abort_flag) : mbar_wait(&ring.full[i], (n / UNITS) & 1, abort_flag);
    Unit t{};
    t.mt = -1;
    if (!there) return t;
    t = read_unit(&ring.unit[i]);
    if (PAIR && rank) mbar_arrive_at(cl_map(smem_u32(&ring.empty[i]), 0));
    else mbar_arrive(&ring.empty[i]);
    return t;
}
template <bool PAIR>
__device__ __forceinline__ bool give_unit(UnitRing& ring, uint32_t n, const Unit& t, volatile int* abort_flag) {
    const uint32_t i = n % UNITS, parity = ((n / UNITS) & 1) ^ 1;
    if (!(PAIR ? mbar_wait_pair(&ring.empty[i], parity, abort_flag) : mbar_wait(&ring.empty[i], parity, abort_flag))) return false;
    write_unit(&ring.unit[i], t);
    if (PAIR) {
        long long v[3];
        memcpy(v, &t, sizeof(t));
        const uint32_t far = cl_map(smem_u32(&ring.unit[i]), 1);
#pragma unroll
        for (int k = 0; k < 3; ++k) asm volatile("st.shared::cluster.b64 [%0], %1;" ::"r"(far + 8 * k), "l"(v[k]) : "memory");
        mbar_arrive_at(cl_map(smem_u32(&ring.full[i]), 1));
    }
    mbar_arrive(&ring.full[i]);
    return true;
}

template <int MODE>
__device__ __forceinline__ int unit_cols(const LossGemm& p, const Unit& t) {   // columns of B that are there
    return MODE == PRODUCTS ? min(p.tn, p.H - t.nt * p.tn) : min(p.tn, p.cols - t.nt * p.tn);
}

// Columns that a product of two CTAs has; each has half of them (products: whole panels of 64).
template <int MODE>
__device__ __forceinline__ int pair_cols(int cols) { return MODE == PRODUCTS ? (cols + 127) / 128 * 128 : (cols + 63) / 64 * 64; }

// 32 columns of an accumulator row: from tensor memory, or from the sums in registers.
template <bool SUMS>
__device__ __forceinline__ void fetch32(float* v, uint32_t taddr, const float* sums, int c) {
    if constexpr (SUMS) {
#pragma unroll
        for (int i = 0; i < 32; ++i) v[i] = sums[c * 32 + i];
    } else {
        tmem_ld32(taddr + c * 32, v);
    }
}

// A row's target distribution, met along its columns (from `col` on, a multiple of 32).  The next two entries of a list are on hand:
// fetching one where it is met took the warp 700 cycles.
template <bool LIST>
struct Targets {
    int next = 0x7fffffff, after = 0x7fffffff, cur = 0, K;
    float q = 1.f, q_after = 0.f;
    const int2* list = nullptr;
    __device__ __forceinline__ Targets(const LossGemm& p, int row, bool there, int col) : K(p.K) {
        if (!there) return;
        if (!LIST) { next = p.target[row]; return; }
        const size_t r = p.src ? p.src[row] : row;
        list = p.list + r * K;
        cur = p.where[r * p.where_ld + (col >> 5)];
        if (cur < K) {
            const int2 a = list[cur];
            next = a.x; q = __int_as_float(a.y);
        }
        fetch_after();
        if (next < col) step();          // (K = 256: `where` says 255 for none)
    }
    __device__ __forceinline__ void fetch_after() {
        after = 0x7fffffff;
        if (cur + 1 < K) {
            const int2 a = list[cur + 1];
            after = a.x; q_after = __int_as_float(a.y);
        }
    }
    __device__ __forceinline__ void step() {
        next = after; q = q_after;
        ++cur;
        fetch_after();
    }
    // f(column, weight) for the targets in [col, col + 32)
    template <typename F>
    __device__ __forceinline__ void in(int col, F f) {
        if (!LIST) {
            if (next >= col && next < col + 32) f(next - col, 1.f);
        } else {
            while (next < col + 32) {
                f(next - col, q);
                step();
            }
        }
    }
};

// What a row's softmax has of some columns: their maximum, the sum of exponentials against it, the targets' weighted logits.
struct RowPart { float m, s, qz; };
__device__ __forceinline__ void join(RowPart& a, float m, float s, float qz) {
    const float m1 = fmaxf(a.m, m), base = m1 == -CUDART_INF_F ? 0.f : m1;
    a.s = a.s * exp2_fast((a.m - base) * kLog2e) + s * exp2_fast((m - base) * kLog2e);
    a.m = m1;
    a.qz += qz;
}

// A row's loss and log-sum-exp.  (Maximum minus the targets' mean logit first: both are large where the logits are.)
__device__ __forceinline__ void row_result(const RowPart& a, int r, const float* ent, float tau, float* loss, float* lse) {
    const float log_s = logf(a.s), ce = (a.m - a.qz) + log_s;
    loss[r] = ent ? tau * tau * (ent[r] + ce) : ce;
    lse[r] = a.m + log_s;
}

// FORWARD epilogue of one row's columns (n_cols of them are outputs) from `col` on.
template <bool LIST, int KIND, int CHUNKS>
__device__ __forceinline__ RowPart forward_row(const LossGemm& p, uint32_t taddr, const float* sums, const float* bias, int col, int n_cols,
                                               Targets<LIST>& targets) {
    RowPart part{-CUDART_INF_F, 0.f, 0.f};
    constexpr bool SUMS = Shape<FORWARD, KIND>::SUMS;
    constexpr int UNROLL = SUMS ? CHUNKS : 1;
#pragma unroll UNROLL
    for (int c = 0; c < CHUNKS; ++c) {
        if (c * 32 >= n_cols) continue;
        float v[32];
        fetch32<SUMS>(v, taddr, sums, c);
        float top[4] = {-CUDART_INF_F, -CUDART_INF_F, -CUDART_INF_F, -CUDART_INF_F};
        const float4* b4 = reinterpret_cast<const float4*>(bias + c * 32);
#pragma unroll
        for (int i = 0; i < 32; i += 4) {
            const float4 b = b4[i / 4];
            const float bb[4] = {b.x, b.y, b.z, b.w};
#pragma unroll
            for (int k = 0; k < 4; ++k) v[i + k] = (v[i + k] + bb[k]) * p.rtau;
#pragma unroll
            for (int k = 0; k < 4; ++k) top[k] = fmaxf(top[k], v[i + k]);
        }
        float qz = 0.f;
        targets.in(col + c * 32, [&](int at, float q) {
            const float z = pick32(v, at);
            if (q != 0.f) qz += q * z;
        });
        const float m = fmaxf(fmaxf(top[0], top[1]), fmaxf(top[2], top[3]));
        const float m1 = fmaxf(part.m, m), base = m1 == -CUDART_INF_F ? 0.f : m1;
        float add[4] = {};
#pragma unroll
        for (int i = 0; i < 32; ++i) add[i & 3] += exp2_fast((v[i] - base) * kLog2e);
        part.s = part.s * exp2_fast((part.m - base) * kLog2e) + ((add[0] + add[1]) + (add[2] + add[3]));
        part.m = m1;
        part.qz += qz;
    }
    return part;
}

// Sums over the 32 lanes of 32 values each: lane l gets the sum of value l.
__device__ __forceinline__ float column_sums(float* v, int lane) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
        const bool up_half = lane & o;
#pragma unroll
        for (int i = 0; i < o; ++i) {
            const float give = up_half ? v[i] : v[i + o], keep = up_half ? v[i + o] : v[i];
            v[i] = keep + __shfl_xor_sync(0xffffffffu, give, o);
        }
    }
    return v[0];
}

// LOGITS epilogue of one row's columns: g, to the next multiple of 64 outputs (K blocks of the product behind), and the warp's share of
// the columns' sums.  bf16: of each 32 columns the first 16 go through 1 KB of shared memory (`stage`; its 16-byte halves swizzled as the
// tensor map says) and out by TMA, the others from registers.  All from registers, 32 rows an instruction, kept the load/store unit busy
// for 4000 cycles a tile; all by TMA, the warp waited for its 1 KB four times a tile (a tile's epilogue: 8600 and 6700 cycles).
template <bool LIST, int KIND, int CHUNKS>
__device__ __forceinline__ void logits_row(const LossGemm& p, const CUtensorMap* map_g, uint8_t* stage, uint32_t taddr, const float* sums, const float* bias,
                                           int g_col, int n_cols, int row, bool there, float scale, float nlse, Targets<LIST>& targets, float* col_sums) {
    const int lane = threadIdx.x & 31, col = p.v0 + g_col;
    __nv_bfloat16* dst = p.g + (size_t)row * p.ldg + g_col;
    const int g_end = (p.cols + 63) / 64 * 64 - g_col;
    constexpr bool SUMS = Shape<LOGITS, KIND>::SUMS;
    constexpr int UNROLL = SUMS ? CHUNKS : 1;
#pragma unroll UNROLL
    for (int c = 0; c < CHUNKS; ++c) {
        if (c * 32 >= n_cols || c * 32 >= g_end) continue;
        float v[32];
        const bool some = col + c * 32 < p.n_out;   // (behind the outputs the accumulator holds what an earlier tile left)
        if (some) {
            fetch32<SUMS>(v, taddr, sums, c);
#pragma unroll
            for (int i = 0; i < 32; i += 4) {
                const float4 b = reinterpret_cast<const float4*>(bias + c * 32)[i / 4];
                const float bb[4] = {b.x, b.y, b.z, b.w};
#pragma unroll
                for (int k = 0; k < 4; ++k) v[i + k] = scale * exp2_fast(((v[i + k] + bb[k]) * p.rtau - nlse) * kLog2e);
            }
            targets.in(col + c * 32, [&](int at, float q) {
#pragma unroll
                for (int i = 0; i < 32; ++i) v[i] = at == i ? v[i] - scale * q : v[i];
            });
        }
        if (!there || !some) {
#pragma unroll
            for (int i = 0; i < 32; ++i) v[i] = 0.f;
        }
        if constexpr (parts_of_g(KIND) == 1) {
            const uint32_t at = smem_u32(stage) + lane * 32, swap = (lane & 4) << 2;
            if (lane == 0) asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory");
            __syncwarp();
#pragma unroll
            for (int k = 0; k < 2; ++k)
                asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(at + ((16u * k) ^ swap)), "r"(pack_bf16x2(v[8 * k], v[8 * k + 1])),
                             "r"(pack_bf16x2(v[8 * k + 2], v[8 * k + 3])), "r"(pack_bf16x2(v[8 * k + 4], v[8 * k + 5])),
                             "r"(pack_bf16x2(v[8 * k + 6], v[8 * k + 7]))
                             : "memory");
            fence_proxy_async();
            __syncwarp();
            if (lane == 0) {
                asm volatile("cp.async.bulk.tensor.2d.global.shared::cta.tile.bulk_group [%0, {%1, %2}], [%3];" ::"l"(reinterpret_cast<uint64_t>(map_g)),
                             "r"(g_col + c * 32), "r"(row), "r"(smem_u32(stage))
                             : "memory");
                asm volatile("cp.async.bulk.commit_group;" ::: "memory");
            }
            store16<1>(dst + c * 32 + 16, 0, v + 16);
        } else {
#pragma unroll
            for (int i = 0; i < 32; i += 16) store16<parts_of_g(KIND)>(dst + c * 32 + i, p.g_plane, v + i);
        }
        if (p.dbp) {
            __syncwarp();
            const float sum = column_sums(v, lane);
            col_sums[c * 32 + lane] = sum;
        }
    }
}

// PRODUCTS epilogue of one row's columns from h0 on; zero: the sum has no term.
// Rows that start anywhere go through the warp's 2 KB of shared memory, 16 columns at a time, and leave two rows an instruction: single
// values straight from registers, 32 rows an instruction, made 0.9 ms of a dW of 52104 x 1429 bf16.
template <int KIND, int CHUNKS>
__device__ __forceinline__ void product_row(const LossGemm& p, const Unit& t, float* stage, uint32_t taddr, const float* sums, int h0, int row, int n_rows,
                                            bool zero) {
    constexpr bool f32 = KIND == F32;
    const bool there = row < (t.dw ? p.cols : n_rows);             // row, of dx: a gathered row; of dW: an output of the piece
    float* slab = t.dw ? p.sdw : p.sdx;
    const int h1 = slab ? p.Hp : p.H;
    uint8_t* out = nullptr;
    float* sum = nullptr;
    if (there) {
        if (slab) sum = slab + ((size_t)t.part * (t.dw ? p.slab_rows_dw : p.Npad) + row) * p.Hp;
        else if (t.dw) out = static_cast<uint8_t*>(p.dw) + (size_t)(p.v0 + row) * p.lddw * (f32 ? 4 : 2);
        else out = static_cast<uint8_t*>(p.dx) + (size_t)p.src[row] * p.lddx * (f32 ? 4 : 2);
    }
    const int vec = t.dw ? p.dw_vec : p.dx_vec;
    constexpr int UNROLL = f32 ? CHUNKS : 1;
#pragma unroll UNROLL
    for (int c = 0; c < CHUNKS; ++c) {
        const int h = h0 + c * 32;
        if (h >= h1) continue;
        float v[32];
        if (zero) {
#pragma unroll
            for (int i = 0; i < 32; ++i) v[i] = 0.f;
        } else fetch32<f32>(v, taddr, sums, c);
        if (!slab && !(vec && h + 32 <= h1)) {
            const int lane = threadIdx.x & 31;
            const unsigned long long mine = reinterpret_cast<unsigned long long>(out);
#pragma unroll
            for (int i0 = 0; i0 < 32; i0 += 16) {
                __syncwarp();
#pragma unroll
                for (int i = 0; i < 16; ++i) stage[lane * 16 + (i ^ (lane & 15))] = v[i0 + i];
                __syncwarp();
                const int col = h + i0 + (lane & 15);
#pragma unroll 4
                for (int r = lane >> 4; r < 32; r += 2) {
                    uint8_t* to = reinterpret_cast<uint8_t*>(__shfl_sync(0xffffffffu, mine, r));
                    const float x = stage[r * 16 + ((lane & 15) ^ (r & 15))];
                    if (to && col < h1) store_one<f32>(to, col, x);
                }
            }
        } else if (!there) {
        } else if (sum) {
            if (!t.dw && p.add_dx) {
                const float4* d = reinterpret_cast<const float4*>(sum + h);
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const float4 b = d[i];
                    v[4 * i] += b.x; v[4 * i + 1] += b.y; v[4 * i + 2] += b.z; v[4 * i + 3] += b.w;
                }
            }
#pragma unroll
            for (int i = 0; i < 32; i += 8) store_sector(sum + h + i, reinterpret_cast<const uint32_t*>(v + i));
        } else if (vec == 2) {
            if constexpr (f32) {
#pragma unroll
                for (int i = 0; i < 32; i += 8) store_sector(reinterpret_cast<float*>(out) + h + i, reinterpret_cast<const uint32_t*>(v + i));
            } else {
#pragma unroll
                for (int i = 0; i < 32; i += 16) store16<1>(reinterpret_cast<__nv_bfloat16*>(out) + h + i, 0, v + i);
            }
        } else {
            if constexpr (f32) {
                float4* d = reinterpret_cast<float4*>(reinterpret_cast<float*>(out) + h);
#pragma unroll
                for (int i = 0; i < 8; ++i) d[i] = make_float4(v[4 * i], v[4 * i + 1], v[4 * i + 2], v[4 * i + 3]);
            } else {
#pragma unroll
                for (int i = 0; i < 32; i += 8) store8<false>(reinterpret_cast<__nv_bfloat16*>(out) + h + i, 0, v + i);
            }
        }
    }
}

template <int MODE, bool LIST, int KIND, bool PAIR>
__global__ void __launch_bounds__((Shape<MODE, KIND>::THREADS), 1)
loss_gemm_kernel(const __grid_constant__ CUtensorMap map_a, const __grid_constant__ CUtensorMap map_b, const __grid_constant__ CUtensorMap map_a2,
                 const __grid_constant__ CUtensorMap map_b2, const LossGemm p) {
    using S = Shape<MODE, KIND>;
    constexpr int TN = S::TN, EPI = S::EPI, A_PARTS = S::A_PARTS, B_PARTS = S::B_PARTS;
    constexpr int TM = PAIR ? 2 * BM : BM;
    extern __shared__ uint8_t smem_raw[];
    __shared__ uint64_t full_bar[kMaxStages], empty_bar[kMaxStages], acc_full[2], acc_empty[2], drain_bar;
    __shared__ UnitRing units;
    __shared__ uint32_t tmem_slot;
    __shared__ int abort_flag;
    __shared__ Unit s_unit[2];
    __shared__ __align__(16) float s_bias[2][TN];
    __shared__ float s_db[MODE == LOGITS ? 4 : 1][TN];                 // [lane quadrant][column of the tile]
    __shared__ float s_part[MODE == FORWARD ? S::GROUPS : 1][3][BM];   // [group][maximum, sum, targets' logits][row]

    const int warp = uniform_warp_index(), lane = threadIdx.x & 31;
    uint8_t* smem = align_smem_1024(smem_raw);
    const uint32_t rank = PAIR ? cl_rank() : 0, cta = PAIR ? blockIdx.x >> 1 : blockIdx.x, ctas = PAIR ? gridDim.x >> 1 : gridDim.x;   // (or pairs)

    if (threadIdx.x == 0) {
        abort_flag = 0;
        auto arrivals = [&](int i, int what) { return 1u + (i == 0 && cta == 0 && p.stall == what); };
        for (int s = 0; s < p.stages; ++s) { mbar_init(&full_bar[s], arrivals(s, 1)); mbar_init(&empty_bar[s], 1); }
        for (int a = 0; a < 2; ++a) { mbar_init(&acc_full[a], arrivals(a, 2)); mbar_init(&acc_empty[a], (PAIR ? 2 : 1) * EPI / 32); }
        for (int i = 0; i < UNITS; ++i) { mbar_init(&units.full[i], arrivals(i, 3)); mbar_init(&units.empty[i], PAIR ? 4 : 2); }
        mbar_init(&drain_bar, 1);
        fence_barrier_init();
        prefetch_tmap(&map_a); prefetch_tmap(&map_b);
        if (MODE != FORWARD) prefetch_tmap(&map_a2);
        if (MODE == PRODUCTS) prefetch_tmap(&map_b2);
    }
    if (warp == 1) {
        if (PAIR) tmem_alloc_pair(&tmem_slot, 512);
        else tmem_alloc(&tmem_slot, 512);
    }
    tc_fence_before();
    __syncthreads();
    if (PAIR) cl_barrier();
    tc_fence_after();
    const uint32_t tmem_base = tmem_slot;
    wait_for_previous();
    const int n_rows = MODE == FORWARD && p.direct ? p.direct : p.ctrl->n_rows;
    const uint32_t n_units = count_units<MODE, TM>(p, n_rows);
    // a short kernel lets the next one start at once; blocks that wait beside a long one slow it (two per cent of a text model's step)
    if (n_units <= ctas) let_next_start();

    const Unit first = unit_of<MODE, TM>(p, n_rows, cta, n_units);

    if (warp == 0) {
        if (elect_one()) {
            int s = 0;
            uint32_t turn = 0;       // of the ring: stage s is used for the (turn + 1)-th time
            uint8_t* a = smem;       // of stage s
            bool ok = true;
            Unit t = first;
            for (uint32_t n = 0; t.mt >= 0; ++n) {
                const uint32_t taken = PAIR && rank ? 0 : p.next ? (uint32_t)atomicAdd(p.next, 1) : n * ctas + cta;   // (there when this unit's first K blocks are under way)
                // The next unit is handed on once the ring is full of this one: at that point nothing waits for this unit's epilogue, which
                // waits for the answer.
                Unit then{};
                auto hand_on = [&] {
                    if (PAIR && rank) {
                        then = next_unit<PAIR>(units, n, rank, &abort_flag);
                        return then.mt >= 0 || !abort_flag;
                    }
                    then = unit_of<MODE, TM>(p, n_rows, ctas + taken, n_units);
                    return give_unit<PAIR>(units, n, then, &abort_flag);
                };
                const int half = PAIR ? pair_cols<MODE>(unit_cols<MODE>(p, t)) / 2 : 0, b0 = rank * half, row0 = t.mt * TM + rank * BM;
                const int panels = PAIR ? half / 64 : (unit_cols<MODE>(p, t) + 63) / 64;
                const bool whole = MODE == PRODUCTS && (t.dw || p.w_panels);      // B's panels by one fetch (of all that a tile may have)
                const int a_part = (MODE == PRODUCTS && t.dw ? BM : p.a_rows) * BK * 2;
                const uint32_t bytes = A_PARTS * a_part + B_PARTS * (MODE == PRODUCTS && !whole ? panels * PANEL_BYTES : p.b_bytes);
                const int hand_at = S::SUMS || (PAIR && rank) ? -1 : t.k0 + min(t.nk, p.stages) - 1;   // (sums, and a pair's other CTA: when it is through)
                for (int kb = t.k0; kb < t.k0 + t.nk; ++kb) {
                    if (!mbar_wait(&empty_bar[s], (turn & 1) ^ 1, &abort_flag)) { ok = false; break; }
                    uint8_t* b = a + A_PARTS * a_part;
                    if (!PAIR || rank == 0) mbar_expect_tx(&full_bar[s], PAIR ? 2 * bytes : bytes);
                    const uint32_t full = PAIR ? cl_map(smem_u32(&full_bar[s]), 0) : 0;
                    auto fetch = [&](uint8_t* to, const CUtensorMap* map, int x, int y, int z) {
                        if (PAIR) tma_load_3d_pair(to, map, x, y, z, full);
                        else tma_load_3d(to, map, x, y, z, &full_bar[s]);
                    };
                    auto fetch4 = [&](uint8_t* to, const CUtensorMap* map, int x, int y, int z, int part) {
                        if (PAIR) tma_load_4d_pair(to, map, x, y, z, part, full);
                        else tma_load_4d(to, map, x, y, z, part, &full_bar[s]);
                    };
                    if (MODE != PRODUCTS || !t.dw) {
                        for (int i = 0; i < A_PARTS; ++i) fetch(a + i * a_part, &map_a, kb * BK, row0, i);
                    } else {
                        for (int i = 0; i < A_PARTS; ++i) fetch4(a + i * a_part, &map_a2, 0, kb * BK, row0 / 64, i);
                    }
                    if (MODE != PRODUCTS) {
                        for (int i = 0; i < B_PARTS; ++i) fetch(b + i * p.b_bytes, &map_b, kb * BK, p.v0 + t.nt * p.tn + b0, i);
                    } else {
                        const int col = t.nt * p.tn + b0, row = t.dw ? kb * BK : p.v0 + kb * BK;
                        const CUtensorMap* map = t.dw ? &map_b2 : &map_b;
                        for (int i = 0; i < B_PARTS; ++i) {
                            if (whole) fetch4(b + i * p.b_bytes, map, 0, row, col / 64, i);
                            else
                                for (int q = 0; q < panels; ++q) fetch4(b + i * p.b_bytes + q * PANEL_BYTES, map, col + q * 64, row, 0, i);
                        }
                    }
                    a += p.stage_bytes;
                    if (++s == p.stages) { s = 0; ++turn; a = smem; }
                    if (kb == hand_at && !hand_on()) { ok = false; break; }
                }
                if (ok && (t.nk == 0 || hand_at < 0)) ok = hand_on();
                if (!ok) break;
                t = then;
            }
            // Copies in flight still write into shared memory (of both CTAs of a pair, which leave together): whoever gave up, and whenever, this
            // thread stays until they are there, or another limit has run out.  (In a normal end there is nothing left to wait for.)
            if (rank == 0) {
                int late = 0;
                for (int i = 0; i < p.stages; ++i) {
                    const uint32_t uses = turn + (i < s);        // of stage i
                    if (uses) mbar_wait(&full_bar[i], (uses - 1) & 1, &late);
                }
            }
        }
    } else if (warp == 1) {
        if (rank == 0 && elect_one()) {
            int s = 0;
            uint32_t turn = 0, n_acc = 0, at = 0;                     // at: of stage s, in units of 16 bytes
            const uint64_t major_k = smem_desc_sw128(smem_u32(smem)), major_mn = smem_desc_mn(smem_u32(smem));
            const uint32_t stage = p.stage_bytes >> 4, b_bytes = p.b_bytes >> 4;
            bool ok = true;
            uint32_t n_unit = 0;
            for (Unit t = first; t.mt >= 0 && ok; t = next_unit<PAIR>(units, n_unit++, 0, &abort_flag)) {
                const int n = PAIR ? pair_cols<MODE>(unit_cols<MODE>(p, t)) : (unit_cols<MODE>(p, t) + 31) / 32 * 32;   // (the epilogues read 32 columns at a time)
                const bool a_mn = MODE == PRODUCTS && t.dw, b_mn = MODE == PRODUCTS;
                const uint32_t idesc = idesc_bf16(TM, n) | (a_mn ? 1u << 15 : 0u) | (b_mn ? 1u << 16 : 0u);
                const uint64_t a_step = a_mn ? 128 : 2, b_step = b_mn ? 128 : 2;   // 16 of K, in units of 16 bytes
                uint32_t tm_d = 0;
                const uint32_t a_part = (MODE == PRODUCTS && t.dw ? BM : p.a_rows) * BK * 2 >> 4;
                const uint64_t a0 = a_mn ? major_mn : major_k, b0 = (b_mn ? major_mn : major_k) + A_PARTS * a_part;
                for (int i = 0; i < t.nk; ++i) {
                    const uint32_t acc = n_acc & 1u;
                    const bool first = i % S::ACC_BLOCKS == 0, last = i % S::ACC_BLOCKS == S::ACC_BLOCKS - 1 || i == t.nk - 1;   // of an accumulator
                    if (first) {
                        const uint32_t parity = ((n_acc >> 1) & 1u) ^ 1u;
                        ok = PAIR ? mbar_wait_pair(&acc_empty[acc], parity, &abort_flag) : mbar_wait(&acc_empty[acc], parity, &abort_flag);
                        if (!ok) break;
                        tm_d = tmem_base + acc * TN;
                    }
                    if (!mbar_wait(&full_bar[s], turn & 1, &abort_flag)) { ok = false; break; }
                    tc_fence_after();
                    const uint64_t adesc = a0 + at, bdesc = b0 + at;
#pragma unroll
                    for (int term = 0; term < S::TERMS; ++term) {
                        const uint64_t ad = adesc + S::a_part(term) * a_part, bd = bdesc + S::b_part(term) * b_bytes;
#pragma unroll
                        for (int k = 0; k < BK / 16; ++k) {
                            if (PAIR) tc_mma_bf16_pair(tm_d, ad + k * a_step, bd + k * b_step, idesc, !first || (term | k) != 0);
                            else tc_mma_bf16(tm_d, ad + k * a_step, bd + k * b_step, idesc, !first || (term | k) != 0);
                        }
                    }
                    if (PAIR) tc_commit_pair(&empty_bar[s]);
                    else tc_commit(&empty_bar[s]);
                    at += stage;
                    if (++s == p.stages) { s = 0; ++turn; at = 0; }
                    if (last) {
                        if (PAIR) tc_commit_pair(&acc_full[acc]);
                        else tc_commit(&acc_full[acc]);
                        ++n_acc;
                    }
                }
            }
            // likewise the products in flight, which read shared memory and write tensor memory
            int late = 0;
            if (PAIR) tc_commit_pair_here(&drain_bar);
            else tc_commit(&drain_bar);
            mbar_wait(&drain_bar, 0, &late);
        }
    } else {
        const int q = warp & 3, group = (warp - 2) >> 2;   // tensor-memory lane quadrant; which columns of the tile
        const int et = threadIdx.x - 64;                   // 0 .. EPI - 1
        const int row_in_tile = q * 32 + lane;
        const int width = group_cols(p.tn, S::GROUPS);
        const int my0 = group * width;                     // first column of this warp's, in the tile
        uint32_t n_acc = 0, n_tile = 0;
        bool ok = true;
        // behind the ring, where a short A is read to no purpose: 16 KB for the epilogue's warps
        uint8_t* stage = smem + (kRingBytes - A_STAGE_BYTES) + (warp - 2) * (32 * A_STAGE_BYTES / EPI);
        Unit then = first;
        for (; then.mt >= 0; ++n_tile) {
            const Unit t = then;
            const uint32_t lanes = tmem_base + my0 + ((uint32_t)(q * 32) << 16);
            const int row = t.mt * TM + rank * BM + row_in_tile;
            float* bias = s_bias[n_tile & 1];
            // what the row needs besides its logits, under way while these are made
            const bool there = row < n_rows;
            const int col = p.v0 + t.nt * p.tn + my0;
            Targets<LIST> targets(p, row, MODE != PRODUCTS && there && my0 < p.tn && col < p.n_out, col);   // (behind the outputs: nothing to find, and no `where`)
            const float scale = MODE == LOGITS && there ? p.scale[row] : 0.f, nlse = MODE == LOGITS && there ? p.nlse[row] : 0.f;
            if (MODE != PRODUCTS && et < p.tn) {
                const int v = p.v0 + t.nt * p.tn + et;         // outputs behind the last one: probability zero
                bias[et] = v < p.n_out ? (p.bias ? p.bias[v] : 0.f) : -CUDART_INF_F;
            }
            // One thread asks for the next unit, which is there before this one's accumulator is; all warps hear the same answer, so that
            // they leave together.  (A warp whose wait runs out goes on without waiting: the others still meet it at the barriers.)
            // With sums it asks when it is through with this one: the operands are not all fetched before that, the accumulators being emptied here.
            auto ask = [&] {
                if (et == 0) write_unit(&s_unit[n_tile & 1], next_unit<PAIR>(units, n_tile, rank, &abort_flag));
                __syncwarp();
                asm volatile("bar.sync 1, %0;" ::"n"(EPI) : "memory");
                then = read_unit(&s_unit[n_tile & 1]);
            };
            if (!S::SUMS) ask();
            else if (MODE != PRODUCTS) {
                __syncwarp();
                asm volatile("bar.sync 1, %0;" ::"n"(EPI) : "memory");
            }
            float sums[S::SUMS ? S::CHUNKS * 32 : 1];
            uint32_t taddr = lanes;
            if constexpr (S::SUMS) {
#pragma unroll
                for (int i = 0; i < S::CHUNKS * 32; ++i) sums[i] = 0.f;
                for (int i = 0; i < t.nk; i += S::ACC_BLOCKS, ++n_acc) {
                    const uint32_t acc = n_acc & 1u;
                    ok = ok && mbar_wait_warp(&acc_full[acc], (n_acc >> 1) & 1u, &abort_flag);
                    __syncwarp();
                    tc_fence_after();
#pragma unroll
                    for (int c = 0; c < S::CHUNKS; ++c) {
                        if constexpr (KIND == BF16_LONG) {
                            // (with 32 values at a time more of the sums go to local memory)
#pragma unroll
                            for (int h = 0; h < 32; h += 16) {
                                float v[16];
                                tmem_ld16(lanes + acc * TN + c * 32 + h, v);
#pragma unroll
                                for (int e = 0; e < 16; ++e) sums[c * 32 + h + e] += v[e];
                            }
                        } else {
                            float v[32];
                            tmem_ld32(lanes + acc * TN + c * 32, v);
#pragma unroll
                            for (int e = 0; e < 32; ++e) sums[c * 32 + e] += v[e];
                        }
                    }
                    tc_fence_before();
                    __syncwarp();
                    if (lane == 0) {
                        if (PAIR && rank) mbar_arrive_at(cl_map(smem_u32(&acc_empty[acc]), 0));
                        else mbar_arrive(&acc_empty[acc]);
                    }
                }
            } else if (t.nk > 0) {
                const uint32_t acc = n_acc & 1u;
                ok = ok && mbar_wait_warp(&acc_full[acc], (n_acc >> 1) & 1u, &abort_flag);
                __syncwarp();
                tc_fence_after();
                taddr = lanes + acc * TN;
            }
            RowPart part{-CUDART_INF_F, 0.f, 0.f};
            if (ok && my0 < p.tn) {
                if constexpr (MODE == FORWARD) {
                    part = forward_row<LIST, KIND, S::CHUNKS>(p, taddr, sums, bias + my0, col, min(width, p.n_out - col), targets);
                } else if constexpr (MODE == LOGITS) {
                    logits_row<LIST, KIND, S::CHUNKS>(p, &map_a2, stage, taddr, sums, bias + my0, t.nt * p.tn + my0, width, row, there, scale, nlse, targets,
                                                      &s_db[q][my0]);
                } else {
                    product_row<KIND, S::CHUNKS>(p, t, reinterpret_cast<float*>(stage), taddr, sums, t.nt * p.tn + my0, row, n_rows, t.nk == 0);
                }
            }
            if (!S::SUMS && t.nk > 0) {
                tc_fence_before();
                __syncwarp();
                if (lane == 0) {
                    if (PAIR && rank) mbar_arrive_at(cl_map(smem_u32(&acc_empty[n_acc & 1u]), 0));
                    else mbar_arrive(&acc_empty[n_acc & 1u]);
                }
                ++n_acc;
            }
            if constexpr (MODE == FORWARD) {
                // the groups' parts of a row become one
                if (group) { s_part[group][0][row_in_tile] = part.m; s_part[group][1][row_in_tile] = part.s; s_part[group][2][row_in_tile] = part.qz; }
                __syncwarp();
                asm volatile("bar.sync 1, %0;" ::"n"(EPI) : "memory");
                if (group == 0 && there) {
#pragma unroll
                    for (int i = 1; i < S::GROUPS; ++i) join(part, s_part[i][0][row_in_tile], s_part[i][1][row_in_tile], s_part[i][2][row_in_tile]);
                    if (p.loss) {
                        row_result(part, p.src[row], p.ent, p.tau, p.loss, p.lse);
                    } else {
                        const size_t at = (size_t)t.nt * p.Npad + row;
                        p.pm[at] = part.m;
                        p.ps[at] = part.s;
                        p.pq[at] = part.qz;
                    }
                }
            }
            if (MODE == LOGITS && p.dbp) {
                __syncwarp();
                asm volatile("bar.sync 1, %0;" ::"n"(EPI) : "memory");
                const int c = t.nt * p.tn + et;
                if (et < p.tn && c < p.cols) p.dbp[(size_t)(t.mt * (TM / BM) + rank) * p.ldg + c] = (s_db[0][et] + s_db[1][et]) + (s_db[2][et] + s_db[3][et]);
            }
            if (S::SUMS) ask();
        }
        if (MODE == LOGITS && parts_of_g(KIND) == 1 && lane == 0) asm volatile("cp.async.bulk.wait_group 0;" ::: "memory");
    }
    __syncwarp();
    tc_fence_before();
    __syncthreads();
    if (PAIR) cl_barrier();     // neither leaves while the other may still reach into its shared memory
    if (warp == 1) {
        tc_fence_after();
        if (PAIR) tmem_dealloc_pair(tmem_base, 512);
        else tmem_dealloc(tmem_base, 512);
    }
    if (threadIdx.x == 0 && abort_flag) p.ctrl->timed_out = kLossTimedOut;
}

// ---------------------------------------------------------------------------
// what is left
// ---------------------------------------------------------------------------
// 8 rows x 32 slices of the partial results a block: eight neighbouring rows are a sector of 32 bytes, and a slice is short (a text
// model's 512 parts: 16 steps; with 32 rows x 8 slices it took 51 us instead of 9).
struct CombineParams {
    LossCtrl* ctrl;
    const int32_t* src; const float *pm, *ps, *pq;
    int parts, Npad;
    const float* ent; float tau;
    float *loss, *lse;
    int direct, n_out; const int32_t* target; const uint8_t* mark;   // direct: rows were not gathered; what they are stands in target or mark
};

__global__ void __launch_bounds__(256) loss_combine_kernel(const CombineParams p) {
    __shared__ float s_m[32][8], s_s[32][8], s_q[32][8];
    let_next_start();
    wait_for_previous();
    const int at_row = threadIdx.x & 7, slice = threadIdx.x >> 3;
    const int j = blockIdx.x * 8 + at_row, n = p.direct ? p.direct : p.ctrl->n_rows;
    if (p.direct && blockIdx.x == 0) {
        const bool bad = __syncthreads_or((int)threadIdx.x < n && mark_of(p.target, p.mark, p.n_out, threadIdx.x) == ROW_BAD);
        if (threadIdx.x == 0) { p.ctrl->status = bad ? WIND_ERR_INVALID_ARG : WIND_OK; p.ctrl->n_rows = n; }
    }
    if ((int)blockIdx.x * 8 >= n) return;
    const float *pm = p.pm, *ps = p.ps, *pq = p.pq;
    float m = -CUDART_INF_F, s = 0.f, qz = 0.f;
    auto add = [&](float m2, float s2) {
        const float m1 = fmaxf(m, m2), base = m1 == -CUDART_INF_F ? 0.f : m1;
        s = s * expf(m - base) + s2 * expf(m2 - base);
        m = m1;
    };
    if (j < n)
#pragma unroll 4
        for (int i = slice; i < p.parts; i += 32) {
            const size_t at = (size_t)i * p.Npad + j;
            add(pm[at], ps[at]);
            qz += pq[at];
        }
    s_m[slice][at_row] = m; s_s[slice][at_row] = s; s_q[slice][at_row] = qz;
    __syncthreads();
    if (threadIdx.x >= 32) return;
    // lane = 8 * quarter + row: eight slices each, then the quarters
    m = -CUDART_INF_F; s = 0.f; qz = 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const int k = (threadIdx.x >> 3) * 8 + i;
        add(s_m[k][at_row], s_s[k][at_row]);
        qz += s_q[k][at_row];
    }
#pragma unroll
    for (int o = 8; o < 32; o <<= 1) {
        add(__shfl_xor_sync(0xffffffffu, m, o), __shfl_xor_sync(0xffffffffu, s, o));
        qz += __shfl_xor_sync(0xffffffffu, qz, o);
    }
    if (threadIdx.x >= 8 || j >= n) return;
    const int r = p.direct ? j : p.src[j];
    const uint8_t mark = p.direct ? mark_of(p.target, p.mark, p.n_out, r) : (uint8_t)ROW_COUNTS;
    if (mark == ROW_COUNTS) {
        row_result(RowPart{m, s, qz}, r, p.ent, p.tau, p.loss, p.lse);
    } else {
        p.loss[r] = p.lse[r] = mark == ROW_BAD ? CUDART_NAN_F : 0.f;
    }
}

// What is left of a piece: partial sums of dW and, behind the last piece, of dx to their places, and db from the row tiles' column sums.
struct FinishParams {
    const LossCtrl* ctrl;
    int H, Hp, blocks_dw, blocks_dx;      // blocks of either; those behind them are db's
    const float* sdw; int s_dw, slab_rows_dw, cols; void* dw; int64_t lddw; int dw_vec;     // dw: of the piece's first output
    const float* sdx; int s_dx, slab_rows_dx; const int32_t* src; void* dx; int64_t lddx; int dx_vec;
    const float* dbp; int ld_dbp; float* db;
};

template <bool F32>
__device__ __forceinline__ void sum_parts(const float* slab, int parts, int slab_rows, int rows, int H, int Hp, const int32_t* src, void* out, int64_t ld,
                                          int vec, int block, int blocks) {
    const int per_row = (H + 3) / 4;
    const long long all = (long long)rows * per_row;
    const size_t stride = (size_t)slab_rows * Hp;
    for (long long i = (long long)block * 256 + threadIdx.x; i < all; i += (long long)blocks * 256) {
        const int r = (int)(i / per_row), h = (int)(i - (long long)r * per_row) * 4;
        const float* at = slab + (size_t)r * Hp + h;
        float4 a = *reinterpret_cast<const float4*>(at);
#pragma unroll 4
        for (int k = 1; k < parts; ++k) {
            const float4 b = *reinterpret_cast<const float4*>(at + k * stride);
            a.x += b.x; a.y += b.y; a.z += b.z; a.w += b.w;
        }
        uint8_t* row = static_cast<uint8_t*>(out) + (size_t)(src ? src[r] : r) * ld * (F32 ? 4 : 2);
        const float v[4] = {a.x, a.y, a.z, a.w};
        if (vec) {
            if (F32) reinterpret_cast<float4*>(row)[h / 4] = a;
            else reinterpret_cast<uint2*>(row)[h / 4] = make_uint2(pack_bf16x2(a.x, a.y), pack_bf16x2(a.z, a.w));
        } else {
#pragma unroll
            for (int k = 0; k < 4; ++k)
                if (h + k < H) store_one<F32>(row, h + k, v[k]);
        }
    }
}

template <bool F32>
__global__ void __launch_bounds__(256) loss_finish_kernel(const FinishParams p) {
    __shared__ float s_sum[8][32];
    let_next_start();
    wait_for_previous();
    const int n_rows = p.ctrl->n_rows;
    int block = blockIdx.x;
    if (block < p.blocks_dw) {
        sum_parts<F32>(p.sdw, p.s_dw, p.slab_rows_dw, p.cols, p.H, p.Hp, nullptr, p.dw, p.lddw, p.dw_vec, block, p.blocks_dw);
        return;
    }
    block -= p.blocks_dw;
    if (block < p.blocks_dx) {
        sum_parts<F32>(p.sdx, p.s_dx, p.slab_rows_dx, n_rows, p.H, p.Hp, p.src, p.dx, p.lddx, p.dx_vec, block, p.blocks_dx);
        return;
    }
    block -= p.blocks_dx;
    const int lane = threadIdx.x & 31, slice = threadIdx.x >> 5, c = block * 32 + lane;     // 32 outputs x 8 slices
    const int tiles = (n_rows + BM - 1) / BM;
    float sum = 0.f;
    if (c < p.cols)
#pragma unroll 4
        for (int i = slice; i < tiles; i += 8) sum += p.dbp[(size_t)i * p.ld_dbp + c];
    s_sum[slice][lane] = sum;
    __syncthreads();
    if (slice || c >= p.cols) return;
    for (int i = 1; i < 8; ++i) sum += s_sum[i][lane];
    p.db[c] = sum;
}

// ---------------------------------------------------------------------------
// host
// ---------------------------------------------------------------------------
// Columns of the tiles of logits.  Narrow ones where wide ones leave SMs idle: the time goes by the CTA with the most tiles, a
// tile's by its columns and (its rows are loaded all the same) by 64 more.
static int tile_cols(int row_tiles, int cols, int most) {
    int best = most;
    long long least = 0;
    if ((long long)row_tiles * cdiv(cols, most) >= kNarrowTiles) return most;
    for (int tn = most; tn >= 64; tn /= 2) {
        const long long time = (((long long)row_tiles * cdiv(cols, tn) + kFillCtas - 1) / kFillCtas) * (tn + 64);
        if (tn == most || time < least) { best = tn; least = time; }
    }
    return best;
}

// Two CTAs to a tile of 256 x 256 fetch a third less from L2 than a CTA to 128 x 256, and draw less power, but there are half as many
// tiles to spread over the chip.  Logits: a text model's step (4096 rows, H = 2048, 65536 outputs) takes 3.50 ms with them and 3.65
// without, the large vocabulary's logits (H = 1024) 102 us either way, the lattice's (H = 640) 30 us against 26.  Products: the large
// vocabulary's 180 us against 189 (8003 rows, 512 tiles), 5 us lost with half the rows, the lattice's 47 us against 38.  (Between
// these widths and numbers of tiles nothing was measured: the borders lie somewhere there.)
static bool pairs_pay(int H, long long tiles) { return H >= 1536 && tiles >= 2 * kFillCtas; }
static bool pairs_pay_products(int H, long long tiles) { return H >= 1024 && tiles >= 3 * kFillCtas; }

LossLayout loss_layout(const wind_output_t& o, int N, int K, int grad, bool most_of_fewer) {
    LossLayout L{};
    const bool f32 = o.dtype == WIND_DT_F32;
    L.planes = f32 ? 3 : 1;
    L.kind = f32 ? F32 : N <= kFineRows ? BF16_FINE : BF16;
    L.g_planes = L.kind;
    L.pack_w = f32 || o.H % 8 || (o.n_out > 1 && (o.ldw % 8 || o.ldw < o.H)) || reinterpret_cast<uintptr_t>(o.w) % 16;
    L.Hp = up(o.H, 64);
    L.Npad = N <= BM ? up(N, BM) : up(N, 2 * BM);
    size_t off = 0;
    auto take = [&](size_t bytes) { size_t at = off; off = align_up(off + bytes); return at; };
    L.ctrl = take(sizeof(LossCtrl));
    const size_t np = (size_t)L.Npad;
    const int most = L.kind == BF16 ? Shape<FORWARD, BF16>::TN : Shape<FORWARD, F32>::TN;
    L.counts = take(N > ROWS_COUNTED ? 4 * (size_t)cdiv(N, ROWS_COUNTED) : 0);
    L.mark = take(K ? np : 0);
    L.src = take(4 * np);
    L.target = take(K ? 0 : 4 * np);
    L.scale = take(grad ? 4 * np : 0);
    L.nlse = take(grad ? 4 * np : 0);
    L.where_ld = up(cdiv(o.n_out, 32), 4);
    L.list = take(8 * (size_t)N * K);
    L.where = take(K ? (size_t)N * L.where_ld : 0);
    L.ent = take(K ? 4 * np : 0);
    L.x = take(2 * (size_t)L.planes * np * L.Hp);
    L.w = take(L.pack_w ? 2 * (size_t)L.planes * o.n_out * L.Hp : 0);
    if (!grad) {
        L.tn = tile_cols(L.Npad / BM, o.n_out, most);
        L.pair = L.kind == BF16 && pairs_pay(o.H, (long long)(L.Npad / BM) * cdiv(o.n_out, 256));
        if (L.pair) L.tn = most;
        L.parts = cdiv(o.n_out, L.tn);
        L.next = take(4);
        size_t parts = (size_t)L.parts * np;
        if (most_of_fewer) parts = std::max((size_t)cdiv(o.n_out, most) * np, std::min((size_t)cdiv(o.n_out, 64) * np, (size_t)kNarrowTiles * (most / 64) * 128));
        L.pm = take(4 * parts);
        L.ps = take(4 * parts);
        L.pq = take(4 * parts);
    } else {
        // a piece: as many outputs as keep its g within kLossPieceBytes, 2048 at least (below that the partial sums of dx, read and
        // written once a piece, cost more than a few per cent of the products)
        const long long all = up(o.n_out, 256);
        const long long fit = (long long)(kLossPieceBytes / (2 * (size_t)L.g_planes * (np ? np : 1))) / 256 * 256;
        L.piece = (int)std::min(all, std::max(2048LL, fit));
        L.pieces = cdiv(o.n_out, L.piece);
        L.tn = tile_cols(L.Npad / BM, std::min(o.n_out, L.piece), most);
        L.pair = L.kind == BF16 && pairs_pay(o.H, (long long)(L.Npad / BM) * cdiv(std::min(o.n_out, L.piece), 256));
        if (L.pair) L.tn = most;
        L.tn_products = f32 ? Shape<PRODUCTS, F32>::TN : Shape<PRODUCTS, BF16>::TN;
        const int ht = cdiv(o.H, L.tn_products), terms = f32 ? 6 : 1;
        const long long t_dx = (long long)(L.Npad / BM) * ht, t_dw = (long long)cdiv(std::min(o.n_out, L.piece), BM) * ht;
        L.pair_products = L.kind == BF16 && pairs_pay_products(o.H, t_dx + t_dw);
        const int kb_dx = cdiv(std::min(o.n_out, L.piece), BK), kb_dw = L.Npad / BK;
        // Parts of a sum: units of at most two thirds of a CTA's share of all K blocks, so that the units taken last fill the gaps, but of
        // 8 K blocks (bf16) at least, and none where the tiles alone are many.
        const int least_kb = cdiv(8, terms);
        // And of at most so many that a bf16 sum stays below kSumAdditions: the tensor cores cut, all one way (2^21 rows of positive
        // activations in one accumulator: dW 0.9 % short).  (fp32 adds each K block up in registers.)
        const int most_kb = f32 ? 1 << 30 : kSumAdditions / (BK / 16) / L.kind;      // (a K block of the FINE kind is two terms long)
        const long long work = t_dx * kb_dx + t_dw * kb_dw, share = (2 * work + 3 * kFillCtas - 1) / (3 * kFillCtas);
        auto parts_of = [&](long long tiles, int kb) {
            const int fill = tiles >= kNarrowTiles ? 1 : cdiv(kb, (int)std::min<long long>(std::max<long long>(share, least_kb), std::max(1, kb)));
            return std::max({1, fill, cdiv(kb, most_kb)});
        };
        L.s_dx = parts_of(t_dx, kb_dx);
        L.s_dw = parts_of(t_dw, kb_dw);
        L.slab_dx = L.s_dx > 1 || L.pieces > 1;
        L.slab_dw = L.s_dw > 1;
        size_t g = (size_t)L.g_planes * np * L.piece, dbp = np / BM * L.piece;
        size_t sdx = L.slab_dx ? (size_t)L.s_dx * np * L.Hp : 0, sdw = L.slab_dw ? (size_t)L.s_dw * up(std::min(o.n_out, L.piece), 128) * L.Hp : 0;
        if (most_of_fewer) {
            // tiles x parts is at most 3/2 kFillCtas (the share of a CTA) more than the tiles, and no part is shorter than least_kb
            auto slab = [&](long long tiles, int kb) {
                return (size_t)std::min(tiles + 3 * kFillCtas / 2, tiles * cdiv(std::max(1, kb), least_kb)) * 128 * std::min(L.tn_products, L.Hp);
            };
            const long long all_dw = (long long)cdiv(o.n_out, 128) * ht;
            sdx = slab(L.pieces > 1 ? t_dx : std::min<long long>(t_dx, kNarrowTiles), kb_dx);
            sdw = slab(std::min<long long>(all_dw, kNarrowTiles), kb_dw);
            if (!f32) {
                // sums cut for their length: parts x rows of dW's slab, where a piece is 2048 outputs or as many as keep g within its limit
                // (4096 at the 65536 rows from which on there are parts), and parts x rows of dx's, where a piece is above 32768 outputs
                const size_t p_dw = cdiv(L.Npad / BK, most_kb), p_dx = cdiv(cdiv(o.n_out, BK), most_kb / 2);
                if (p_dw > 1) sdw = std::max(sdw, std::min(p_dw * up(o.n_out, 128), std::max<size_t>(p_dw * 2048, 8192)) * L.Hp);
                if (p_dx > 1) sdx = std::max(sdx, std::min<size_t>(p_dx * np, 8192) * L.Hp);
            }
            const size_t whole = np * (size_t)all, limit = kLossPieceBytes / 2;
            g = std::min((size_t)L.planes * whole, std::max(limit, (size_t)L.planes * np * 2048));
            if (!f32) g = std::max(g, std::min<size_t>(2 * std::min(np, (size_t)256) * all, std::max(limit, 2 * std::min(np, (size_t)256) * 2048)));
            dbp = std::min(whole, std::max(limit, np * 2048)) / BM;
        }
        L.next = take(4 * 2 * (size_t)(most_of_fewer ? cdiv(o.n_out, 2048) : L.pieces));
        L.g = take(2 * g);
        L.dbp = take(4 * dbp);
        L.sdx = take(4 * sdx);
        L.sdw = take(4 * sdw);
    }
    L.total = off;
    return L;
}

static PFN_cuTensorMapEncodeTiled g_encode_loss = nullptr;
static std::mutex g_loss_mutex;

static cudaError_t get_encode_loss() {
    std::lock_guard<std::mutex> lock(g_loss_mutex);
    if (g_encode_loss) return cudaSuccess;
    void* fn = nullptr;
    cudaDriverEntryPointQueryResult q;
    cudaError_t e = cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &fn, cudaEnableDefault, &q);
    if (e != cudaSuccess) return e;
    if (q != cudaDriverEntryPointSuccess || !fn) return cudaErrorNotSupported;
    g_encode_loss = reinterpret_cast<PFN_cuTensorMapEncodeTiled>(fn);
    return cudaSuccess;
}

// bf16 [planes][rows][cols], rows `ld` elements apart, box = 64 columns x box_rows rows, 128-byte swizzle, zero fill outside
static cudaError_t loss_map(CUtensorMap* map, const void* base, uint64_t planes, uint64_t rows, uint64_t cols, uint64_t ld, uint32_t box_rows) {
    cuuint64_t dims[3] = {cols, rows, planes};
    cuuint64_t strides[2] = {ld * 2, rows * ld * 2};
    cuuint32_t box[3] = {(cuuint32_t)BK, box_rows, 1};
    cuuint32_t estr[3] = {1, 1, 1};
    CUresult r = g_encode_loss(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, const_cast<void*>(base), dims, strides, box, estr,
                               CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                               CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    return r == CUDA_SUCCESS ? cudaSuccess : cudaErrorInvalidValue;
}

typedef void (*LossKernel)(const CUtensorMap, const CUtensorMap, const CUtensorMap, const CUtensorMap, const LossGemm);

// The same matrix as groups of 64 columns, so that one fetch brings a K block of `panels` of them, each as the MN-major descriptors want it:
// [parts][cols / 64][rows][64], box = 64 columns x 64 rows x panels.  With a fetch for each panel a text
// model's products took 1477 us instead of 1430.  one_group: cols need not be whole groups; boxes of one panel, by column.
static cudaError_t panel_map(CUtensorMap* map, const void* base, uint64_t parts, uint64_t rows, uint64_t cols, uint64_t ld, uint32_t panels, bool one_group) {
    cuuint64_t dims[4] = {one_group ? cols : 64, rows, one_group ? 1 : cols / 64, parts};
    cuuint64_t strides[3] = {ld * 2, 128, rows * ld * 2};
    cuuint32_t box[4] = {64, 64, one_group ? 1 : panels, 1};
    cuuint32_t estr[4] = {1, 1, 1, 1};
    CUresult r = g_encode_loss(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 4, const_cast<void*>(base), dims, strides, box, estr,
                               CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                               CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    return r == CUDA_SUCCESS ? cudaSuccess : cudaErrorInvalidValue;
}

// where the tiles of logits store g (its first part): boxes of 16 columns x 32 rows
static cudaError_t store_map(CUtensorMap* map, void* base, uint64_t rows, uint64_t cols) {
    cuuint64_t dims[2] = {cols, rows};
    cuuint64_t strides[1] = {cols * 2};
    cuuint32_t box[2] = {16, 32};
    cuuint32_t estr[2] = {1, 1};
    CUresult r = g_encode_loss(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, base, dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
                               CU_TENSOR_MAP_SWIZZLE_32B, CU_TENSOR_MAP_L2_PROMOTION_NONE, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    return r == CUDA_SUCCESS ? cudaSuccess : cudaErrorInvalidValue;
}

template <int MODE, int KIND, bool PAIR>
static LossKernel loss_kernel_of(bool list) {
    return list && MODE != PRODUCTS ? loss_gemm_kernel<MODE, MODE != PRODUCTS, KIND, PAIR> : loss_gemm_kernel<MODE, false, KIND, PAIR>;
}
struct LossLaunch { LossKernel kernel; int threads, a_parts, b_parts, pair; };
template <int MODE>
static LossLaunch loss_launch_of(bool list, int kind, bool pair) {
    if (kind == F32) return {loss_kernel_of<MODE, F32, false>(list), Shape<MODE, F32>::THREADS, Shape<MODE, F32>::A_PARTS, Shape<MODE, F32>::B_PARTS, 0};
    if (kind == BF16_FINE) return {loss_kernel_of<MODE, BF16_FINE, false>(list), Shape<MODE, BF16_FINE>::THREADS, Shape<MODE, BF16_FINE>::A_PARTS, 1, 0};
    if constexpr (MODE != PRODUCTS)
        if (kind == BF16_LONG)
            return {pair ? loss_kernel_of<MODE, BF16_LONG, true>(list) : loss_kernel_of<MODE, BF16_LONG, false>(list), Shape<MODE, BF16_LONG>::THREADS, 1, 1, pair};
    return {pair ? loss_kernel_of<MODE, BF16, true>(list) : loss_kernel_of<MODE, BF16, false>(list), Shape<MODE, BF16>::THREADS, 1, 1, pair};
}

// Shared-memory opt-in of the kernels of this file.
static cudaError_t loss_set_attributes() {
    static bool done_on[64] = {};   // the attribute belongs to the (function, device) pair
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    if (dev < 0 || dev >= 64) return cudaErrorInvalidDevice;
    std::lock_guard<std::mutex> lock(g_loss_mutex);
    if (done_on[dev]) return cudaSuccess;
    for (int list = 0; list < 2; ++list)
        for (int kind = BF16; kind <= BF16_LONG; ++kind)
            for (const bool pair : {false, true})
                for (const LossLaunch& l : {loss_launch_of<FORWARD>(list, kind, pair), loss_launch_of<LOGITS>(list, kind, pair), loss_launch_of<PRODUCTS>(list, kind, pair)})
                    if ((e = cudaFuncSetAttribute(l.kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kRingBytes + 1024)) != cudaSuccess) return e;
    done_on[dev] = true;
    return cudaSuccess;
}

static int vec_rows(const void* p, int64_t ld, int H, bool f32) {   // accesses of rows of H elements: 0 single, 1 of 16 bytes, 2 of 32
    const uintptr_t at = reinterpret_cast<uintptr_t>(p) | (uintptr_t)(ld * (f32 ? 4 : 2));
    return H % 8 || at % 16 ? 0 : at % 32 ? 1 : 2;
}

// (every kernel here waits for the one before it ahead of its first access to memory)
template <typename... Params, typename... Args>
static cudaError_t launch_small(void (*kernel)(Params...), int blocks, cudaStream_t stream, const Args&... args) {
    static_assert(sizeof...(Params) == sizeof...(Args), "");
    return [&](Params... typed) {
        void* list[] = {(void*)&typed...};
        return launch_overlapped((const void*)kernel, dim3((unsigned)blocks), dim3(256), list, 0, stream);
    }(args...);
}

// The ring of K blocks in shared memory.  A stage holds what is fetched: a_rows rows of A (few, where the call has few: the products
// read 128, and what lies behind the a_rows makes rows of the result that nobody looks at) and a tile's columns of B.  A call of one
// row has 16 K blocks of 64 columns under way instead of four.
static void ring_of(LossGemm& p, const LossLaunch& l, int a_rows, int tn) {
    p.a_rows = a_rows;
    p.b_bytes = (l.pair ? tn / 2 : tn) * BK * 2;
    p.stage_bytes = l.a_parts * a_rows * BK * 2 + l.b_parts * p.b_bytes;
    p.stages = std::min(kMaxStages, (kRingBytes - A_STAGE_BYTES) / p.stage_bytes);
}

static cudaError_t launch_gemm(const LossLaunch& l, long long units, int sms, const CUtensorMap& a, const CUtensorMap& b, const CUtensorMap& a2,
                               const CUtensorMap& b2, const LossGemm& p, cudaStream_t stream) {
    void* args[5] = {(void*)&a, (void*)&b, (void*)&a2, (void*)&b2, (void*)&p};
    if (!l.pair)
        return launch_overlapped((const void*)l.kernel, dim3((unsigned)std::min<long long>(units, sms)), dim3(l.threads), args, kRingBytes + 1024, stream);
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3(2 * (unsigned)std::min<long long>(units, sms / 2)); cfg.blockDim = dim3(l.threads); cfg.dynamicSmemBytes = kRingBytes + 1024; cfg.stream = stream;
    cudaLaunchAttribute at[2];
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[0].val.programmaticStreamSerializationAllowed = 1;
    at[1].id = cudaLaunchAttributeClusterDimension;
    at[1].val.clusterDim.x = 2; at[1].val.clusterDim.y = 1; at[1].val.clusterDim.z = 1;
    cfg.attrs = at;
    cfg.numAttrs = 2;
    return cudaLaunchKernelExC(&cfg, (const void*)l.kernel, args);
}

static std::atomic<int> g_loss_stall{0};   // 0, or 3 x kernel + wait
int loss_set_stall(int which) { return g_loss_stall.exchange(which >= 1 && which <= 9 ? which : 0); }
static int stall_of(LossMode mode) {
    const int which = g_loss_stall.load() - 3 * mode;
    return which >= 1 && which <= 3 ? which : 0;
}

cudaError_t loss_run(const LossCall& c) {
    const LossLayout& L = c.lay;
    const bool f32 = c.o.dtype == WIND_DT_F32;
    const size_t es = f32 ? 4 : 2;
    // tensor maps need the device's context in this thread; a stream's flags, which see to that, may not be asked for in a capture
    cudaStreamCaptureStatus capture = cudaStreamCaptureStatusNone;
    cudaError_t e = cudaStreamIsCapturing(c.stream, &capture);
    if (e == cudaSuccess && capture == cudaStreamCaptureStatusNone) e = bind_context(c.stream);
    if (e != cudaSuccess) return e;
    LossCtrl* ctrl = reinterpret_cast<LossCtrl*>(c.ws + L.ctrl);
    if (c.N == 0) {   // no rows: no loss, no gradient
        e = cudaMemsetAsync(ctrl, 0, offsetof(LossCtrl, timed_out), c.stream);
        if (e == cudaSuccess && c.grad && c.dw) e = cudaMemset2DAsync(c.dw, (size_t)c.lddw * es, 0, (size_t)c.o.H * es, (size_t)c.o.n_out, c.stream);
        if (e == cudaSuccess && c.grad && c.db) e = cudaMemsetAsync(c.db, 0, 4 * (size_t)c.o.n_out, c.stream);
        return e;
    }
    if ((e = get_encode_loss()) != cudaSuccess) return e;
    if ((e = loss_set_attributes()) != cudaSuccess) return e;
    int sms = 0;
    if ((e = loop_sm_count(&sms)) != cudaSuccess) return e;

    RowsParams r{};
    r.ctrl = ctrl;
    r.N = c.N; r.n_out = c.o.n_out; r.K = c.K; r.H = c.o.H; r.Hp = L.Hp; r.Npad = L.Npad; r.grad = c.grad;
    r.x_vec = vec_rows(c.x, c.ldx, c.o.H, f32);
    r.dx_vec = vec_rows(c.dx, c.lddx, c.o.H, f32);
    r.tau = c.tau;
    r.target = c.target; r.ids = c.ids; r.y = c.y; r.x = c.x; r.ldx = c.ldx;
    r.counts = reinterpret_cast<int32_t*>(c.ws + L.counts);
    r.mark = c.ws + L.mark;
    r.next = reinterpret_cast<int32_t*>(c.ws + L.next);
    r.n_next = c.grad ? 2 * L.pieces : 1;
    r.src = reinterpret_cast<int32_t*>(c.ws + L.src);
    r.target_c = reinterpret_cast<int32_t*>(c.ws + L.target);
    r.scale_c = reinterpret_cast<float*>(c.ws + L.scale);
    r.nlse_c = reinterpret_cast<float*>(c.ws + L.nlse);
    r.list = reinterpret_cast<int2*>(c.ws + L.list);
    r.where = c.ws + L.where;
    r.where_ld = L.where_ld;
    r.ent = reinterpret_cast<float*>(c.ws + L.ent);
    r.xc = reinterpret_cast<__nv_bfloat16*>(c.ws + L.x);
    r.loss = c.loss; r.lse_out = c.lse_out; r.lse = c.lse; r.dloss = c.dloss; r.dx = c.dx; r.lddx = c.lddx;
    if (c.K) {
        void (*list)(RowsParams) = c.K <= 32 ? loss_list_kernel<1> : c.K <= 64 ? loss_list_kernel<2> : c.K <= 128 ? loss_list_kernel<4> : loss_list_kernel<8>;
        if ((e = launch_small(list, cdiv(c.N, 8), c.stream, r)) != cudaSuccess) return e;
    }
    r.counted = c.N > ROWS_COUNTED;
    if (r.counted) {
        if ((e = launch_small(loss_count_kernel, cdiv(c.N, ROWS_COUNTED), c.stream, r)) != cudaSuccess) return e;
    }
    // Two blocks an SM, while they are not too long: each counts the rows before its own (20011 rows of H = 640: 11.5 us; with 4 to 6 an SM
    // 12 to 14, with one of 1024 threads 11.3; with x fetched before counting the same)
    r.per_block = std::min(256, up(cdiv(c.N, 2 * sms), 8));
    r.row_blocks = cdiv(c.N, r.per_block);
    const void* w = c.o.w;
    int64_t ldw = c.o.ldw;
    int w_cols = c.o.H, pack_blocks = 0;
    if (L.pack_w) {
        r.w = w; r.ldw = ldw; r.w_vec = vec_rows(w, ldw, c.o.H, f32);
        r.wc = reinterpret_cast<__nv_bfloat16*>(c.ws + L.w);
        pack_blocks = (int)std::min<long long>(((long long)c.o.n_out * (L.Hp / 8) + 255) / 256, 8LL * sms);
        w = r.wc; ldw = L.Hp; w_cols = L.Hp;
    }
    const bool one_tile = L.Npad == BM;      // of rows: then the tiles of logits write db themselves
    if (c.grad && one_tile) r.db = c.db;
    if (c.grad) r.dw = c.dw;
    // A loss of one row tile, whose x TMA can start on, needs no gathering (rows of padding are left out at the end): a launch less, and
    // 11 us instead of 14 for one row against 8193 outputs.
    const bool direct = !c.grad && one_tile && !L.pack_w && r.x_vec && (c.N == 1 || c.ldx >= c.o.H);
    if (!direct && (e = launch_small(f32 ? loss_gather_kernel<true> : loss_gather_kernel<false>, r.row_blocks + pack_blocks, c.stream, r)) != cudaSuccess)
        return e;

    LossGemm p{};
    p.ctrl = ctrl;
    p.n_out = c.o.n_out; p.H = c.o.H; p.Hp = L.Hp; p.Npad = L.Npad; p.K = c.K;
    p.kb = L.Hp / BK;
    p.tn = L.tn;
    p.rtau = 1.f / c.tau;
    p.bias = c.o.b;
    p.src = r.src; p.target = r.target_c; p.list = r.list; p.where = r.where; p.where_ld = r.where_ld;
    const int few = std::min(BM, up(c.N, 8));    // rows of A that a fetch brings
    CUtensorMap map_x, map_w, map_w64, map_x64, map_g, map_g64, map_store{};
    if (direct) e = loss_map(&map_x, c.x, 1, c.N, c.o.H, c.N == 1 ? c.o.H : c.ldx, few);
    else e = loss_map(&map_x, r.xc, L.planes, L.Npad, L.Hp, L.Hp, few);
    if (e != cudaSuccess) return e;
    if ((e = loss_map(&map_w, w, L.planes, c.o.n_out, w_cols, ldw, L.pair ? L.tn / 2 : L.tn)) != cudaSuccess) return e;
    const int logits_kind = L.kind == BF16 && p.kb > kLongBlocks ? BF16_LONG : L.kind;
    const int row_tiles = L.Npad / BM;
    const long long logit_rows = L.pair ? row_tiles / 2 : row_tiles;    // tiles
    if (!c.grad) {
        p.v0 = 0; p.cols = c.o.n_out; p.n_vt = cdiv(c.o.n_out, L.tn);
        p.pm = reinterpret_cast<float*>(c.ws + L.pm);
        p.ps = reinterpret_cast<float*>(c.ws + L.ps);
        p.pq = reinterpret_cast<float*>(c.ws + L.pq);
        const LossLaunch l = loss_launch_of<FORWARD>(c.K > 0, logits_kind, L.pair);
        ring_of(p, l, few, L.tn);
        p.next = direct ? nullptr : r.next;
        if (direct) { p.direct = c.N; p.src = nullptr; p.target = c.target; }
        const bool final = !direct && L.parts == 1;     // (no launch for joining what is one part)
        if (final) { p.loss = c.loss; p.lse = c.lse_out; p.ent = c.K ? r.ent : nullptr; p.tau = c.tau; }
        p.stall = stall_of(FORWARD);
        if ((e = launch_gemm(l, logit_rows * p.n_vt, sms, map_x, map_w, map_x, map_w, p, c.stream)) != cudaSuccess) return e;
        if (final) return cudaSuccess;
        CombineParams q{};
        q.ctrl = ctrl; q.src = r.src; q.pm = p.pm; q.ps = p.ps; q.pq = p.pq; q.parts = L.parts; q.Npad = L.Npad;
        q.ent = c.K ? r.ent : nullptr; q.tau = c.tau; q.loss = c.loss; q.lse = c.lse_out;
        q.direct = p.direct; q.n_out = c.o.n_out; q.target = c.target; q.mark = c.K ? r.mark : nullptr;
        return launch_small(loss_combine_kernel, cdiv(c.N, 8), c.stream, q);
    }

    p.scale = r.scale_c; p.nlse = r.nlse_c;
    p.g = reinterpret_cast<__nv_bfloat16*>(c.ws + L.g);
    p.ldg = L.piece; p.g_plane = (size_t)L.Npad * L.piece;
    p.ht = cdiv(c.o.H, L.tn_products); p.s_dx = L.s_dx; p.s_dw = L.s_dw;
    p.sdx = L.slab_dx ? reinterpret_cast<float*>(c.ws + L.sdx) : nullptr;
    p.sdw = L.slab_dw ? reinterpret_cast<float*>(c.ws + L.sdw) : nullptr;
    p.slab_rows_dw = up(std::min(c.o.n_out, L.piece), 128);
    p.dx_first = cdiv(cdiv(std::min(c.o.n_out, L.piece), BK), L.s_dx) >= cdiv(L.Npad / BK, L.s_dw);
    p.dx = c.dx; p.lddx = c.lddx; p.want_dx = c.dx != nullptr; p.dx_vec = vec_rows(c.dx, c.lddx, c.o.H, f32);
    p.dw = c.dw; p.lddw = c.lddw; p.want_dw = c.dw != nullptr; p.dw_vec = vec_rows(c.dw, c.lddw, c.o.H, f32);
    if ((e = loss_map(&map_g, p.g, L.g_planes, L.Npad, L.piece, L.piece, few)) != cudaSuccess) return e;
    const uint32_t panels = (L.pair_products ? L.tn_products / 2 : L.tn_products) / 64;
    p.w_panels = w_cols % 64 == 0;
    if ((e = panel_map(&map_g64, p.g, L.g_planes, L.Npad, L.piece, L.piece, BM / 64, false)) != cudaSuccess) return e;
    if ((e = store_map(&map_store, p.g, L.Npad, L.piece)) != cudaSuccess) return e;
    if ((e = panel_map(&map_x64, r.xc, L.planes, L.Npad, L.Hp, L.Hp, panels, false)) != cudaSuccess) return e;
    if ((e = panel_map(&map_w64, w, L.planes, c.o.n_out, w_cols, ldw, panels, !p.w_panels)) != cudaSuccess) return e;
    for (int piece = 0; piece < L.pieces; ++piece) {
        p.v0 = piece * L.piece;
        p.cols = std::min(L.piece, c.o.n_out - p.v0);
        p.tn = L.tn;
        p.n_vt = cdiv(p.cols, L.tn);
        p.add_dx = piece > 0;
        p.dbp = !c.db ? nullptr : one_tile ? c.db + p.v0 : reinterpret_cast<float*>(c.ws + L.dbp);
        const LossLaunch l = loss_launch_of<LOGITS>(c.K > 0, logits_kind, L.pair);
        ring_of(p, l, few, L.tn);
        p.next = r.next + 2 * piece;
        p.stall = stall_of(LOGITS);
        if ((e = launch_gemm(l, logit_rows * p.n_vt, sms, map_x, map_w, map_store, map_w, p, c.stream)) != cudaSuccess) return e;
        FinishParams f{};
        f.ctrl = ctrl; f.H = c.o.H; f.Hp = L.Hp; f.cols = p.cols;
        int finish_blocks = 0;
        if (c.db && !one_tile) {
            f.dbp = p.dbp; f.ld_dbp = L.piece; f.db = c.db + p.v0;
            finish_blocks = cdiv(p.cols, 32);
        }
        p.tn = L.tn_products;
        const LossLaunch lp = loss_launch_of<PRODUCTS>(false, L.kind, L.pair_products);
        ring_of(p, lp, c.dw ? BM : few, p.tn);
        p.a_rows = few;
        const int tm = lp.pair ? 2 * BM : BM;
        const long long units = (c.dx ? (long long)L.s_dx * (L.Npad / tm) * p.ht : 0) + (c.dw ? (long long)L.s_dw * cdiv(p.cols, tm) * p.ht : 0);
        p.next = r.next + 2 * piece + 1;
        p.stall = stall_of(PRODUCTS);
        if (units && (e = launch_gemm(lp, units, sms, map_g, map_w64, map_g64, map_x64, p, c.stream)) != cudaSuccess) return e;
        if (c.dw && L.slab_dw) {
            f.sdw = p.sdw; f.s_dw = L.s_dw; f.slab_rows_dw = p.slab_rows_dw;
            f.dw = static_cast<uint8_t*>(c.dw) + (size_t)p.v0 * c.lddw * es; f.lddw = c.lddw; f.dw_vec = p.dw_vec;
            f.blocks_dw = (int)std::min<long long>(((long long)p.cols * ((c.o.H + 3) / 4) + 255) / 256, 8LL * sms);
        }
        if (c.dx && L.slab_dx && piece == L.pieces - 1) {
            f.sdx = p.sdx; f.s_dx = L.s_dx; f.slab_rows_dx = L.Npad;
            f.src = r.src; f.dx = c.dx; f.lddx = c.lddx; f.dx_vec = p.dx_vec;
            f.blocks_dx = (int)std::min<long long>(((long long)c.N * ((c.o.H + 3) / 4) + 255) / 256, 8LL * sms);
        }
        finish_blocks += f.blocks_dw + f.blocks_dx;
        if (finish_blocks && (e = launch_small(f32 ? loss_finish_kernel<true> : loss_finish_kernel<false>, finish_blocks, c.stream, f)) != cudaSuccess) return e;
    }
    return cudaSuccess;
}

}  // namespace wind
