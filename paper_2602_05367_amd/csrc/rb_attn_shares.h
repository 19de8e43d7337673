// How attention of few new tokens over a cache is cut into shares: arithmetic on whole numbers alone, the same on any machine.
//
// The arrays first and lengths are a caller's, read on the device.  Sums over arrays that are not in order can have any value, wrapped around 32 bits; what follows
// from them here stays among the sequences, their rows and the shares all the same.
#pragma once

namespace rb {
namespace attn {

// positions of a sequence in a cache: what its length says, as far as the page table reaches
__device__ __forceinline__ int positions(int length, int width, int page_shift)
{
    return min(max(length, 0), (int)min((long long)width << page_shift, 0x7fffffc0ll));
}

namespace few {

constexpr int KEYS = 32, ROWS = 32;

// Where the work of a sequence lies among all tiles of a key head.  (All of them, as many as rows and positions allow, are counted in 31 bits: see few_applies.)
struct Shape {
    static constexpr int JOB = ROWS;
    int rows, blocks, tiles;
    __device__ __forceinline__ int count() const { return blocks * tiles; }
    template <class Args> static __device__ __forceinline__ Shape of(const Args &A, int q0, int q1, int length)
    {
        q0 = min(max(q0, 0), A.tokens_q);
        q1 = min(max(q1, q0), A.tokens_q);
        const int rows = (q1 - q0) * A.group;
        // a sequence that has rows but no positions: one tile, of which they see nothing
        return {rows, (rows + ROWS - 1) / ROWS, rows ? max((positions(length, A.width, A.page_shift) + KEYS - 1) / KEYS, 1) : 0};
    }
};

// All tiles in equal shares, the first ones longer by one; never more shares than tiles: none is empty
struct Shares {
    int n, each, longer;
    __device__ __forceinline__ Shares(int all, int wavefronts) : n(min(wavefronts, max(all, 1))), each((int)((unsigned)all / (unsigned)n)), longer((int)((unsigned)all % (unsigned)n)) {}
    __device__ __forceinline__ int start(int w) const { return w * each + min(w, longer); }
    __device__ __forceinline__ int of(int tile) const
    {
        const unsigned in_longer = (unsigned)(each + 1) * longer;
        return (unsigned)tile < in_longer ? (int)((unsigned)tile / (unsigned)(each + 1)) : longer + (int)(((unsigned)tile - in_longer) / (unsigned)each);
    }
    // the first and last share that have some of `tiles` tiles from `from` on; false: these are not among all
    __device__ __forceinline__ bool of_job(int from, int tiles, int &first, int &last) const
    {
        if (from < 0 || each < 1) return false;
        first = of(from), last = of((int)((unsigned)from + (unsigned)tiles - 1u));
        return first >= 0 && first <= last && last < n;
    }
};

// A position in the row of tiles.  entries(s, q0, q1, length): what the arrays say of a sequence
struct Cursor {
    int s, block, t;
    Shape shape;
    int q0, n_k;
    template <class Args> __device__ __forceinline__ bool there(const Args &A) const { return s < A.n_seqs; }
    template <class Args, class Entries> __device__ __forceinline__ void visit(const Args &A, Entries entries)      // sequence s, or nothing behind the last
    {
        if (!there(A)) {
            shape = {0, 1, 0x7fffffff};
            n_k = 0;
            return;
        }
        int from, to, length;
        entries(s, from, to, length);
        q0 = min(max(from, 0), A.tokens_q);
        shape = Shape::of(A, from, to, length);
        n_k = positions(length, A.width, A.page_shift);
    }
    // at tile `tile` of sequence s; false: there is no such
    template <class Args, class Entries> __device__ __forceinline__ bool stand(const Args &A, int tile, Entries entries)
    {
        if (s < 0 || !there(A)) return false;
        visit(A, entries);
        if (tile < 0 || shape.blocks == 0) return false;
        block = min((int)((unsigned)tile / (unsigned)shape.tiles), shape.blocks - 1);
        t = min(tile - block * shape.tiles, shape.tiles - 1);
        return true;
    }
    template <class Args, class Entries> __device__ __forceinline__ void advance(const Args &A, Entries entries)
    {
        if (++t < shape.tiles) return;
        t = 0;
        if (++block < shape.blocks) return;
        block = 0;
        do {
            ++s;
            visit(A, entries);
        } while (shape.blocks == 0);
    }
};

}  // namespace few
}  // namespace attn
}  // namespace rb
