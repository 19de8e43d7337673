// Shares of the attention of few new tokens over a cache, run on the CPU: arrays in order are cut as defined, and whatever the arrays hold, every part lies in
// the workspace and every row that is read among the queries.
#include <algorithm>
#include <climits>
#include <cstdint>
#include <cstdio>
#include <cstdlib>
#include <random>
#include <vector>

#define __forceinline__ inline
static inline int min(int a, int b) { return a < b ? a : b; }
static inline int max(int a, int b) { return a > b ? a : b; }
static inline long long min(long long a, long long b) { return a < b ? a : b; }
#include "rb_attn_shares.h"

using namespace rb::attn::few;

struct Args {
    int n_seqs, tokens_q, group, width, page_shift;
};

#define CHECK(x) \
    do { \
        if (!(x)) { \
            std::printf("trial %d: %s\n", trial, #x); \
            std::exit(1); \
        } \
    } while (0)

int main()
{
    std::mt19937 rng(17);
    auto any = [&](int lo, int hi) { return std::uniform_int_distribution<int>(lo, hi)(rng); };
    long long wrapped = 0, jobs = 0, steps = 0;
    for (int trial = 0; trial < 4000; ++trial) {
        const bool in_order = trial % 4 == 0;
        Args A;
        A.n_seqs = trial % 3 ? any(1, 300) : any(1, 5);
        A.group = 1 << any(0, 4);
        A.tokens_q = max(1, any(1, 32 * A.n_seqs) / A.group);
        A.page_shift = any(3, 16);
        A.width = in_order ? any(1, 300) : any(1, max(1, (int)(32ll * (0x7fffffffll / (2 * A.n_seqs + 2) - 2) >> A.page_shift)));
        const int wavefronts = 4 * any(1, 256);
        std::vector<int> first(A.n_seqs + 1), lengths(A.n_seqs);
        if (in_order) {
            for (int i = 1; i < A.n_seqs; ++i) first[i] = any(0, A.tokens_q);
            first[A.n_seqs] = A.tokens_q;
            std::sort(first.begin(), first.end());
            for (int &l : lengths) l = any(0, A.width << A.page_shift);
        } else {
            const int kind = any(0, 3);
            for (int i = 0; i <= A.n_seqs; ++i)
                first[i] = kind == 0 ? (i % 2 ? A.tokens_q : 0) : kind == 1 ? (int)rng() : any(0, 7) ? any(0, A.tokens_q) : any(0, 1) ? INT_MIN : INT_MAX;
            for (int &l : lengths) l = kind == 0 || any(0, 3) == 0 ? INT_MAX : (int)rng();
        }
        auto entries = [&](int s, int &q0, int &q1, int &length) {
            CHECK(s >= 0 && s < A.n_seqs);
            q0 = first[s], q1 = first[s + 1], length = lengths[s];
        };
        std::vector<uint32_t> before(A.n_seqs + 1, 0u);      // sums as 32 bits have them
        long long real = 0;
        for (int s = 0; s < A.n_seqs; ++s) {
            const int count = Shape::of(A, first[s], first[s + 1], lengths[s]).count();
            before[s + 1] = before[s] + (uint32_t)count;
            real += count;
        }
        wrapped += real > INT_MAX;
        CHECK(!in_order || real <= INT_MAX);
        const int all = (int)before[A.n_seqs];
        const Shares shares(all, wavefronts);
        CHECK(!in_order || !all || (shares.start(0) == 0 && shares.start(shares.n) == all && shares.n <= wavefronts));
        // the join: every job of every sequence
        for (int s = 0; s < A.n_seqs; ++s) {
            const Shape shape = Shape::of(A, first[s], first[s + 1], lengths[s]);
            for (int b = 0; b < shape.blocks; b += 1 + shape.blocks / 5) {
                const int from = (int)(before[s] + (uint32_t)b * shape.tiles);
                int w0 = -1, w1 = -1;
                const bool there = shares.of_job(from, shape.tiles, w0, w1);
                CHECK(!there || (w0 >= 0 && w0 <= w1 && w1 < wavefronts));
                if (in_order) CHECK(there && shares.start(w0) <= from && from < shares.start(w0 + 1) && shares.start(w1) < from + shape.tiles && from + shape.tiles <= shares.start(w1 + 1));
                ++jobs;
            }
        }
        // the wavefronts: from where the sums say, or from anywhere
        for (int i = 0; i < 8; ++i) {
            const int w = any(0, shares.n - 1), begin = shares.start(w), n = shares.start(w + 1) - begin;
            if (n <= 0) continue;
            Cursor at = {};
            int tile = begin;
            if (in_order || i % 2) {
                while (at.s < A.n_seqs && (int)before[at.s + 1] <= begin) ++at.s;
                if (at.there(A)) tile = (int)((uint32_t)begin - before[at.s]);
            } else {
                at.s = any(-1, A.n_seqs), tile = (int)rng();
            }
            const bool stands = at.stand(A, tile, entries);
            CHECK(stands || !in_order);
            if (!stands) continue;
            for (int k = 0; k < min(n, 3000) && at.there(A); ++k, ++steps) {
                CHECK(at.shape.rows > 0 && at.block >= 0 && at.block < at.shape.blocks && at.t >= 0 && at.t < at.shape.tiles);
                const int row0 = at.block * ROWS, last = min(row0 + ROWS - 1, at.shape.rows - 1);
                CHECK(row0 < at.shape.rows && at.q0 >= 0 && at.q0 + last / A.group < A.tokens_q);
                if (in_order) CHECK((uint32_t)(begin + k) == before[at.s] + (uint32_t)(at.block * at.shape.tiles + at.t));
                at.advance(A, entries);
            }
        }
    }
    if (!wrapped) return 1;
    std::printf("%lld jobs and %lld steps in range, %lld sums wrapped\n", jobs, steps, wrapped);
    return 0;
}
