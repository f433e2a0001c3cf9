// Internal declarations of the operators of hybrid layers: whole prompts, and layers with a state of fixed size per
// sequence (short convolution, selective scan).  Not part of the public ABI.
#pragma once

#include "internal.h"

namespace ap {

// ---- device work lists (all int32, uploaded as one blob per plan) ---------

// Rows of one sequence that a block walks: a whole sequence of a state plan, or a piece of it.
struct StateUnit {
    int32_t row0;        // first row
    int32_t rows;        // rows of the unit (>= 1)
    int32_t slot;        // the sequence's slot
    int32_t flags;
    int32_t seg_first;   // scan: workspace entry of the sequence's first piece
    int32_t seg;         // scan: number of the piece
    int32_t seq_rows;    // rows of the whole sequence
    int32_t pad;
};
static_assert(sizeof(StateUnit) == 32, "StateUnit layout");
enum : int32_t {
    kUnitFirst = 1,      // the sequence's first rows are among the unit's
    kUnitLast = 2,       // its last rows are
    kUnitKept = 4,       // the sequence goes on from its slot (else: from zeros)
    kUnitStateOnly = 8,  // scan: only the state behind the piece is wanted
};

// One unit of prompt attention on the tensor cores: 128 consecutive rows of a prompt for one or two q heads of a kv head.
struct PromptTile {
    int32_t row0;        // first query row
    int32_t rows;        // 1..128
    int32_t start;       // first row of the prompt
    int32_t q_head;
    int32_t q_head_b;    // second q head of the same kv head sharing the K/V stream, or -1
    int32_t kv_head;
    int32_t pad[2];
};
static_assert(sizeof(PromptTile) == 32, "PromptTile layout");

// One unit of the kernel for short prompts (and one kv head): blocks of 16 rows of a prompt.
struct ShortPrompt {
    int32_t start;       // first row of the prompt
    int32_t rows;        // rows of the prompt
    int32_t block0, block1;
};
static_assert(sizeof(ShortPrompt) == 16, "ShortPrompt layout");

}  // namespace ap

namespace ap {
struct PromptLists {              // units of prompt attention, block i's from begin[i] to begin[i + 1]
    const PromptTile *tiles = nullptr;
    const int32_t *begin = nullptr;
    int blocks = 0;
};
}  // namespace ap

struct ap_prompt_plan {
    ap_kv_pool *pool = nullptr;
    ap::PlanBuffer buf{};
    int num_q_heads = 0;
    float scale = 0.f;
    ap_prompt_info info{};
    ap::PromptLists lists[2];     // units of one tile, of two
    const ap::ShortPrompt *d_short = nullptr;
};

struct ap_state_pool {
    ap_state_desc desc{};
    bool owns_conv = false, owns_scan = false;
    int sm_count = 0;
    std::vector<ap::PlanBuffer> plan_buffers;     // recycled plan staging
};

struct ap_state_plan {
    ap_state_pool *pool = nullptr;
    ap_state_desc desc{};         // of the pool: any pool of the same shape will do
    ap::PlanBuffer buf{};
    ap_state_info info{};
    size_t workspace_bytes = 0;
    int n_conv = 0;               // units of the convolution: runs of rows
    int n_first = 0, n_second = 0;   // units of the scan's first launch, of its second
    int n_single = 0;             // sequences with one row
    const ap::StateUnit *d_conv = nullptr, *d_first = nullptr, *d_second = nullptr, *d_single = nullptr;
};

namespace ap {

constexpr int kConvThreads = 128; // each takes 4 channels
constexpr int kScanTile = 32;     // pieces of a sequence are multiples of it, as it is of the rows that the scan stages at a time

struct ScanArgs {                 // by value to the kernels
    const uint16_t *x, *dt, *b, *c, *z;       // bf16
    const float *a, *d_skip, *dt_bias;
    uint16_t *out;
    float *state;                 // scan plane
    float *seg_state;             // [pieces][channels][state_dim]: the state behind a piece begun from zeros (the first: from its start)
    float *seg_dt;                // [pieces][channels]: sum of the piece's steps
    int64_t xs, dts, bs, cs, zs, os;
    int channels, softplus;
};

int scan_warp_channels(int state_dim);        // channels that a warp of the scan takes
cudaError_t launch_conv(const ap_state_pool *pool, const ap_state_plan *plan, const ap_conv_desc &conv, cudaStream_t stream);
cudaError_t launch_scan(const ap_state_pool *pool, const ap_state_plan *plan, const ScanArgs &args, cudaStream_t stream);
cudaError_t launch_prompt(ap_kv_pool *pool, const ap_prompt_plan *plan, const void *q, const void *k, const void *v,
                          void *out, float *lse, const ap_prompt_strides &strides, cudaStream_t stream);

// rows of [n_rows][heads][head_dim] bf16, `row_stride` elements apart: box of 128 rows of a head (see tensor_map.cu)
int encode_rows_tensor_map(CUtensorMap *map, const void *base, int64_t n_rows, int heads, int head_dim, int64_t row_stride);

}  // namespace ap
