// Products C = A B^T in 16 bits, several in one launch, sums split where their
// tiles leave SMs without work.
#pragma once

#include "tiles.cuh"

namespace ifvs {

// A K-major [rows][K] or MN-major [K][rows]; B the same with `cols`.  Up to three
// products in one launch, items (tiles, or parts of a tile's sum) in their order.
struct Product {
    CUtensorMap a, b, c;
    Grid g;
    int splits;          // parts of the sum; more than one: float32 parts in `parts`, added by k_join_parts
    int items;           // tiles x splits
    bool a_mn, b_mn;
    float* parts;        // [splits][rows][cols]
};
// Sums over the rows of a matrix (a bias's gradient), made by the warps that would wait for
// the first tile: CTA c adds part c mod n_parts of the rows in every n_phases-th block of 256
// columns from c / n_parts on.
struct RowSums {
    const void* from;    // [rows][cols], or null: none
    int64_t rows;
    int cols, n_parts, n_phases;
    float* parts;        // [n_parts][cols]
};
struct Products {
    Product p[3];
    int n, items;
    RowSums sums;
};

// C = the sum of the parts, in order; up to three products and the sums
struct Parts {
    const float* parts[4];
    void* c[4];
    int64_t n[4];        // values, a multiple of 8
    int splits[4];
    int sums;            // which of them are the row sums, or -1
};

// Products of one launch, in the order they are added
struct Plan {
    const TileArgs a;
    bool pairs;          // 256 x 256 tiles of CTA pairs; else 128 x 128
    uint8_t* work;       // for parts of sums
    Products all;
    Parts parts;
    int joined = 0;
    cudaError_t e = cudaSuccess;
    explicit Plan(const TileArgs& a_, bool pairs_, uint8_t* work_) : a(a_), pairs(pairs_), work(work_) {
        all.n = all.items = 0;
        all.sums.from = nullptr;
        parts.sums = -1;
    }

    int rows_tile() const { return pairs ? 256 : 128; }
    // C [rows][cols] = A B^T over K
    void add(int64_t rows, int64_t cols, int64_t K, const void* A, bool a_mn, const void* B, bool b_mn, void* C) {
        Product& p = all.p[all.n++];
        auto then = [&](cudaError_t r) { e = e == cudaSuccess ? r : e; };
        then(a_mn ? make_map(&p.a, a.type, A, K, rows, rows, 64) : make_map(&p.a, a.type, A, rows, K, K, kRows));
        then(b_mn ? make_map(&p.b, a.type, B, K, cols, cols, 64) : make_map(&p.b, a.type, B, cols, K, K, 128));
        then(make_map(&p.c, a.type, C, rows, cols, cols, 32));
        p.g = Grid{ceil_div(rows, rows_tile()), ceil_div(cols, rows_tile()), ceil_div(K, kStepK), (int)rows, (int)cols};
        p.a_mn = a_mn;
        p.b_mn = b_mn;
        p.splits = splits_of(a, rows, cols, K, pairs);
        p.items = p.g.m_tiles * p.g.n_tiles * p.splits;
        p.parts = nullptr;
        all.items += p.items;
        if (p.splits > 1) {
            p.parts = (float*)work;
            work += (size_t)p.splits * rows * cols * sizeof(float);
            parts.parts[joined] = p.parts;
            parts.c[joined] = C;
            parts.n[joined] = rows * cols;
            parts.splits[joined++] = p.splits;
        }
    }
    // After the products are added: `out` [cols], the sums over the rows of `from`
    void add_sums(const void* from, int64_t rows, int cols, void* out) {
        const int ctas = grid(), blocks = ceil_div(cols, 256);
        int phases = ctas / 16 < blocks ? ctas / 16 : blocks;
        if (phases < 1) phases = 1;
        all.sums = RowSums{from, rows, cols, ctas / phases, phases, (float*)work};
        parts.parts[joined] = (float*)work;
        parts.c[joined] = out;
        parts.n[joined] = cols;
        parts.sums = joined;
        parts.splits[joined++] = ctas / phases;
        work += (size_t)(ctas / phases) * cols * sizeof(float);
    }
    static size_t sums_bytes(const TileArgs& a, int cols) { return (size_t)a.num_sms * cols * sizeof(float); }
    // CTAs of the launch
    int grid() const {
        const int64_t most = a.num_sms / (pairs ? 2 : 1);
        return (int)(all.items < most ? all.items : most) * (pairs ? 2 : 1);
    }
    // Parts of a tile's sum: where the tiles leave SMs without work, at least four
    // stages each.  A sum of any length is cut below 2^16 stages, which bounds
    // every wait for a tile.
    static int splits_of(const TileArgs& a, int64_t rows, int64_t cols, int64_t K, bool pairs) {
        const int tile = pairs ? 256 : 128, steps = ceil_div(K, kStepK);
        const int64_t tiles = (int64_t)ceil_div(rows, tile) * ceil_div(cols, tile), slots = a.num_sms / (pairs ? 2 : 1);
        int64_t n = slots / tiles;
        if (n > steps / 4) n = steps / 4;
        if (n > 32) n = 32;
        const int64_t least = ((int64_t)steps + 65535) / 65536;
        return (int)(n > least ? n : (least > 1 ? least : 1));
    }
    static size_t part_bytes(const TileArgs& a, int64_t rows, int64_t cols, int64_t K, bool pairs) {
        const int n = splits_of(a, rows, cols, K, pairs);
        return n > 1 ? (size_t)n * rows * cols * sizeof(float) : 0;
    }
    cudaError_t launch(bool chain, cudaStream_t s);
};

}  // namespace ifvs
