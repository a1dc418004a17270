// Between pconv_linear.hip (entry points, plans, sums of parts) and the products' translation units, one per storage type.
#pragma once

#include <cstddef>

namespace pconv {

// What is done with a product's result R[i][j] before it is stored.
struct Finish {
    int kind;                   // kForward, kGradInput, kFloat
    int act, first;             // first: the residual goes in front of the activation
    const float* bias;          // kForward: float[J] or null
    const void* add;            // kForward: residual, kGradInput: add; or null
    long long ld_add;
    const void* zin;            // kGradInput: the activation's argument, or null
    long long ld_zin;
    void* z;                    // kForward: z, or null
    void* out;                  // storage type, kFloat: float
    long long ld_out;           // also of z
};
enum { kForward = 0, kGradInput = 1, kFloat = 2 };

// Column sums that were taken over strips of rows and are still to be added: out[j] = sum of parts[strip][j].  parts null: none
struct Strips {
    const float* parts;
    int strips, N;
    float* out;
};

// R[i][j] = sum over c of A(i, c) * B(j, c).  A(i, c) is at a[i * lda + c] or, a_rows, at a[c * lda + i]; B alike.
struct Product {
    const void* a;
    const void* b;
    long long lda, ldb;         // elements
    int I, J, C;
    bool a_rows, b_rows;
    Finish f;
    int tile;                   // kTiles index
    int splits, c_per;          // workgroups that share a tile, and the c each takes (a multiple of a stage's)
    float* parts;               // splits > 1: [splits][I][J] partial sums
    Strips strips;              // added in the launch that adds the parts (splits > 1)
};

constexpr int kComputeUnits = 256;          // of an MI355X: plans and workspaces are the same whatever device is current
constexpr int kTiles = 3;
constexpr int kTileEdges[kTiles] = {256, 128, 64};
constexpr int kStageBytes = 128;            // of c per stage, of one row

int launch_product_f32(const Product& p, void* stream);
int launch_product_f16(const Product& p, void* stream);
int launch_product_bf16(const Product& p, void* stream);

// The product for few rows of x (I <= kFewRows), forward only: see few_rows_kernel.
constexpr int kFewRows = 16;
int launch_few_rows_f32(const Product& p, void* stream);
int launch_few_rows_f16(const Product& p, void* stream);
int launch_few_rows_bf16(const Product& p, void* stream);

}  // namespace pconv
