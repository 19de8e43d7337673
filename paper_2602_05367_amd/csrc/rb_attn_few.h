// What the two kernels for few new tokens share, over a cache of 16 bits (rb_attn_few.hip) and of 8 (rb_attn_few8.hip): how parts of a job lie in the workspace, and are joined.
#pragma once
#include <algorithm>

#include "rb_attn.h"
#include "rb_attn_host.h"
#include "rb_attn_shares.h"

namespace rb {
namespace attn {
namespace few {

constexpr int WAVES = 4;

// the part that share w has of a job of which it does not have all: its first job (0) or its last (1)
template <int D> __device__ __forceinline__ PartOfRows<D, ROWS> part_of(Address workspace, int kvh, int wavefronts, int w, int which)
{
    return PartOfRows<D, ROWS>(workspace, ((size_t)kvh * wavefronts + w) * 2 + which);
}

// A job that several wavefronts had parts of
template <class T, int D> __global__ __launch_bounds__(256) void join_kernel(const Args A, int wavefronts, int joined)
{
    const int lane = threadIdx.x & 63, kvh = blockIdx.x % A.kv_heads, block = blockIdx.x / A.kv_heads, row0 = blockIdx.y * joined;
    const int *first = global_at<const int>(A.first_q), *lengths = global_at<const int>(A.first_k);
    const Sums<Shape> sums_of(A, first, lengths, lane);
    const int s = __builtin_amdgcn_readfirstlane(sums_of.of_block(block));
    int q0, q1, length;
    sums_of.entries(s, q0, q1, length);
    const Shape shape = Shape::of(A, q0, q1, length);
    const int b = block - block_start(q0, s, A.group, ROWS);
    if (b < 0 || b >= shape.blocks || b * ROWS + row0 >= shape.rows) return;
    const Shares shares(sums_of.before(A.n_seqs), wavefronts);
    const int from = sums_of.before(s) + b * shape.tiles;
    int w0, w1;
    if (!shares.of_job(from, shape.tiles, w0, w1) || w0 == w1) return;      // (one: it has stored the result)
    const bool starts_inside = shares.start(w0) < from;      // the first part is that share's last, all others are their shares' first
    const int n_q = shape.rows / A.group, n_k = positions(length, A.width, A.page_shift);
    q0 = min(max(q0, 0), A.tokens_q);
    auto token = [&](int r) { return (b * ROWS + r) / A.group; };
    join_rows<T, D>(
        joined, w1 - w0 + 1, row0, min(shape.rows - b * ROWS - row0, joined), A.dim,
        [&](int i) { return part_of<D>(A.parts, kvh, wavefronts, w0 + i, i == 0 && starts_inside ? 1 : 0); },
        [&](int r) { return global_at<uint8_t>(A.o) + ((long long)(q0 + token(r)) * A.heads + kvh * A.group + (b * ROWS + r) % A.group) * (A.dim * 2); },
        [&](int r) { return n_k - n_q + token(r) < 0; });
}

// The launches of a call: a kernel by `groups` workgroups per key head, start(grid, threads), and the join
template <class T, int D, class Start> int launch(const Args &A, int groups, hipStream_t stream, Start start)
{
    const long long jobs = attn::block_numbers(A.tokens_q, A.n_seqs, A.group, ROWS) * A.kv_heads;
    if (!one_launch(jobs, 256)) return RB_ERR_SHAPE;      // (many more sequences than the search for one is made for)
    start(dim3((unsigned)(groups * A.kv_heads)), dim3(64 * WAVES));
    const int rows = (int)std::min((long long)ROWS, (long long)A.tokens_q * A.group), joined = rows_joined(jobs, rows);      // rows of one job, at most
    hipLaunchKernelGGL((join_kernel<T, D>), dim3((unsigned)jobs, (rows + joined - 1) / joined), dim3(256), 0, stream, A, groups * WAVES, joined);
    return hipGetLastError() == hipSuccess ? RB_OK : RB_ERR_HIP;
}
inline size_t workspace_bytes(int kv_heads, int dim, int groups)
{
    return (size_t)kv_heads * groups * WAVES * 2 * (dim <= 64 ? PartOfRows<64, ROWS>::FLOATS : PartOfRows<128, ROWS>::FLOATS) * 4;
}

}  // namespace few
}  // namespace attn
}  // namespace rb
