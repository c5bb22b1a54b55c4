// Parameter blocks and launchers shared between the kernel files and the C-ABI host code.
#pragma once

#include <cuda.h>

#include "tempo_common.cuh"

namespace tempo {

struct DispatchParams {
  int T, k, E, G_max, R_max, M_cap;
  const int32_t* topk_ids;
  const int32_t* n_valid;
  const int32_t* replica_map;
  const int32_t* quota;
  uint32_t* cum_counts;
  int32_t* counts;
  int32_t* inst_count;
  int32_t* inst_off;
  int32_t* pair_row;
  int32_t* row_pair;
  int32_t* tile_inst;
  int32_t* m_pad;
  uint32_t* status;
  int max_m;   // 0: instances follow each other in whole tiles; M > 0: masked layout, instance i owns rows [i*M, (i+1)*M)
};
size_t dispatch_smem_bytes(int E, int R, int G);

struct SampledParams {
  int T, k, E, G_max, R_max, M_cap;
  const int32_t* topk_ids;
  const int32_t* n_valid;
  const int32_t* replica_map;
  const float* table;
  unsigned long long seed;
  uint32_t layer;
  uint32_t* cum_counts;
  int32_t* counts;
  int32_t* inst_count;
  int32_t* inst_off;
  int32_t* pair_row;
  int32_t* row_pair;
  int32_t* tile_inst;
  int32_t* m_pad;
  uint32_t* status;
};
size_t dispatch_sampled_smem_bytes(int E, int R, int G);
cudaError_t launch_count_dispatch_sampled(const SampledParams& p, cudaStream_t stream);
cudaError_t launch_count_dispatch(const DispatchParams& p, cudaStream_t stream);

struct PermuteParams {
  int k, d, M_cap;
  const __nv_bfloat16* x;
  const int32_t* row_pair;
  int T;                      // token rows (token-major form only)
  const int32_t* pair_row;    // NULL: row-major form (gather per row); else token-major form (quantise once per token)
  const int32_t* tile_inst;   // masked layout only (else NULL): tiles with -1 hold no rows and are left alone
  const int32_t* m_pad;
  uint8_t* a_q;
  uint8_t* a_sf;
};
cudaError_t launch_permute_pad(const PermuteParams& p, int num_sms, cudaStream_t stream);
cudaError_t launch_permute_pad_bf16(const PermuteParams& p, __nv_bfloat16* a, int num_sms, cudaStream_t stream);

struct QuantizeParams {
  int T, d;
  int sf_stride;              // bytes per token of x_sf: 4 * ceil((d / 128) / 4)
  const __nv_bfloat16* x;
  const int32_t* n_valid;
  uint8_t* x_q;
  uint8_t* x_sf;
};
cudaError_t launch_quantize_tokens(const QuantizeParams& p, int num_sms, cudaStream_t stream);

struct CombineParams {
  int T, k, d;
  const __nv_bfloat16* y;
  const int32_t* pair_row;
  const float* topk_w;
  const int32_t* n_valid;
  __nv_bfloat16* out;
};
cudaError_t launch_combine(const CombineParams& p, cudaStream_t stream);

struct PackLayout {
  size_t off_w13, off_w2, off_sf13, off_sf2, total;
  int J1, J2, NT1, NT2;
};
PackLayout pack_layout(int G, int d, int f);
PackLayout pack_layout_bf16(int G, int d, int f);   // off_w13, off_w2, NT1, NT2, total only
cudaError_t launch_pack_bf16(int G, int d, int f, const __nv_bfloat16* w13, const __nv_bfloat16* w2, uint8_t* packed,
                             cudaStream_t stream);
cudaError_t launch_pack(int G, int d, int f, const uint8_t* w13_q, const float* w13_s, const uint8_t* w2_q,
                        const float* w2_s, uint8_t* packed, uint32_t* status, cudaStream_t stream);

// One of the two GEMMs of the FFN as the fused kernel sees it.
struct GemmSide {
  int Kb;        // K / 128
  int JK;        // scale atoms along K = ceil(Kb / 4)
  int NT;        // 256-column tiles per instance
  const uint8_t* wt;     // packed B tiles, 32 KB each, [inst][nt][kb]
  const uint8_t* sfa;    // scale atoms of the A operand
  const uint8_t* sfb;    // scale atoms of the packed weights
};

struct FfnParams {
  GemmSide side[2];      // 0: gate/up (A = a_q), 1: down (A = h_q)
  int run_mask;          // bit 0: run the gate/up tiles, bit 1: run the down tiles
  int G_max, M_cap;
  int d, f;
  int J_h;               // scale atoms along f of the H buffer
  const int32_t* inst_off;
  const int32_t* m_pad;
  // masked layout (stride_tiles > 0): instance i owns the M-tiles [i*stride_tiles, (i+1)*stride_tiles) and
  // uses the first ceil(inst_count[i]/128) of them; inst_off and m_pad are not read
  int stride_tiles;
  const int32_t* inst_count;
  uint8_t* h_q;
  uint8_t* h_sf;
  __nv_bfloat16* y;
  // gather form (ffn_kernel<false, true>): the gate/up operand rows are fetched from the per-token buffers
  const uint8_t* x_q;        // e4m3 codes [T, d]
  const uint8_t* x_sf;       // scale bytes [T, x_sf_stride]
  const int32_t* row_pair;   // row -> pair (token = pair / k), -1: zero row
  int x_sf_stride, k, T;
  int32_t* ready;        // workspace: per M-tile, epilogue warps of finished gate/up tiles
  int32_t* done;         // workspace: per M-tile, down tiles that have seen `ready` complete
  uint32_t* status;
  unsigned long long wait_ns;   // bound of every device-side wait of the kernel, in nanoseconds
};
size_t ffn_workspace_bytes(int M_cap);
// The bf16 variant: Kb counts 64-value K-blocks, the scale pointers and J_h are unused, h_q holds bf16.
cudaError_t launch_ffn_bf16(const CUtensorMap& tmA1, const CUtensorMap& tmA2, const CUtensorMap& tmY,
                            const FfnParams& p, int num_sms, cudaStream_t stream);
cudaError_t launch_ffn(const CUtensorMap& tmA1, const CUtensorMap& tmA2, const CUtensorMap& tmY,
                       const FfnParams& p, int num_sms, cudaStream_t stream);
cudaError_t launch_ffn_gather(const CUtensorMap& tmA2, const CUtensorMap& tmY, const FfnParams& p, int num_sms,
                              cudaStream_t stream);

// ---- around the block, and the layer for a few tokens -------------------------------------------------
struct NormParams {
  int T, d, layer;           // layer: subtract the row's mean
  int stream_f32, param_f32, gate_f32, gate_vec;   // gate_vec: the gate's row can be read with the row's vectors
  bool shift;                // eight columns at a time at any alignment (norm_shifts)
  bool param_vec;            // the weights and biases can be read in 16-byte loads
  const __nv_bfloat16* y;    // NULL: the norm before a block
  const void* r;
  const void* post_w;
  const void* post_b;
  const void* gate;
  const void* next_w;
  const void* next_b;
  const int32_t* n_valid;
  void* r_out;
  __nv_bfloat16* x;
  size_t ld_y, ld_r, ld_r_out, ld_x, gate_row, gate_col;
  float eps, r_scale, y_scale;
};
bool norm_shifts(const NormParams& p, int vec);
cudaError_t launch_norm(const NormParams& p, int vec, int num_sms, cudaStream_t stream);

struct RoutePlan {
  int E16, tile_rows, x_box, w_box, w_boxes, stage_bytes, stages, splits, ctas;
};
struct RouteParams {
  int T, k, E, Kb;           // Kb = d / 64
  int sigmoid, renormalise;
  float scale;
  const float* bias;
  const int32_t* n_valid;
  int32_t* ids;
  float* w;
  uint32_t* status;
  int E16, tile_rows, x_box, w_box, w_boxes, stage_bytes, stages, splits, tmem_cols, pitch;   // from the plan
};
RoutePlan route_plan(int T, int E, int d, int num_sms);
cudaError_t launch_route(const CUtensorMap& tmX, const CUtensorMap& tmW, RouteParams p, const RoutePlan& r, cudaStream_t stream);

constexpr int kFewMaxT = 64, kFewMaxPairs = 1024;
constexpr int kFewMaxSms = 160;      // the workspace is sized for so many CTAs, whatever the device
constexpr int kFewSplit = 4;         // most partial sums of a (256 output columns, expert) line of the down product
struct FewLayout {
  int counter_ints;                  // of one of the two counter sets
  size_t off_leave, off_counters, off_x, off_h, off_gu, off_y, total;
};
struct FewParams {
  int T, k, E, R, G, d;
  int Kb1, Kb2, NT1, NT2, J1, J2;    // K-blocks, column blocks and scale atoms of the gate/up and the down product
  const int32_t* ids;
  const float* w;
  const int32_t* n_valid;
  const int32_t* replica_map;
  const __nv_bfloat16* x;
  const uint8_t* w13;
  const uint8_t* w2;
  const uint8_t* sf13;
  const uint8_t* sf2;
  unsigned int* leave;
  int32_t* counters;
  int counter_ints;
  uint8_t* x_img;
  uint8_t* h_img;
  float* gu_part;
  float* y_part;
  __nv_bfloat16* out;
  uint32_t* status;
  unsigned long long wait_ns;
  int stages, stage_bytes, slots;    // set by the launcher
};
FewLayout few_layout(int T, int k, int G, int d, int f, int num_sms);
cudaError_t launch_few(const FewParams& p, bool bf16, int num_sms, cudaStream_t stream);

// ---- the attention half of a layer ---------------------------------------------------------------------
struct HeadsParams {
  int T, Hq, Hkv, D, rot, interleaved, n_pos, w_f32;
  bool q_vec, k_vec, v_vec, q_out_vec, k_out_vec, w_vec;   // eight elements can be read or written as 16 bytes
  bool quads;                // rows and angles can be read four elements at a time, pairs in fours
  bool rot_vec;              // a lane's eight elements turn with one other lane's (or among themselves), angles in 16-byte loads
  const __nv_bfloat16* q;
  const __nv_bfloat16* k;
  const __nv_bfloat16* v;
  const void* q_w;
  const void* k_w;
  const int32_t* positions;
  const float* cos_sin;
  const int32_t* n_valid;
  __nv_bfloat16* q_out;
  __nv_bfloat16* k_out;
  size_t ld_q, hd_q, ld_k, hd_k, ld_v, hd_v, ld_q_out, hd_q_out, ld_k_out, hd_k_out;
  float eps, inverse_d;
  uint32_t* status;
  int n_pages, page_size;    // append only, as all below
  const int32_t* slots;
  uint8_t* cache;
  uint32_t k_blocks;         // set by the launcher: blocks that take keys
  int rounds;                // and how often a group of lanes takes its number of query heads
};
cudaError_t launch_heads(const HeadsParams& p, bool append, int num_sms, cudaStream_t stream);

struct KvReadParams {
  int n, n_pages, page_size, Hkv;
  const uint8_t* cache;
  const int32_t* slots;
  __half* k;
  __half* v;
  uint32_t* status;
};
cudaError_t launch_kv_read(const KvReadParams& p, int D, cudaStream_t stream);

constexpr int kAttendMaxB = 1024;
constexpr int kAttendMaxSms = 160;   // the workspace is sized for so many CTAs, whatever the device
constexpr int kAttendManyRows = 256; // rows of an item in the kernel for many queries
struct AttendLayout {
  size_t off_counters, off_groups, off_stats, off_out, total;
};
AttendLayout attend_layout(int D);
struct AttendParams {
  int B, T, Hkv, group;      // group: query heads of a key head
  int max_pages, page_size, page_shift, n_pages;
  bool wide;                 // rows of q and out can be read and written 32 bytes at a time
  int rows_few, len_few;    // sequences of up to so many rows (queries times group) or tokens are the few-query kernel's
  const __nv_bfloat16* q;
  const uint8_t* cache;
  const int32_t* page_table;
  const int32_t* lens;
  const int32_t* q_start;
  const int32_t* n_valid;
  __nv_bfloat16* out;
  size_t ld_q, hd_q, ld_out, hd_out;
  float scale_log2;          // scale * log2(e)
  uint32_t* status;
  unsigned int* counters;    // arrivals of the CTAs that share an item, by the first of them; zero between calls
  unsigned int* groups;      // and of a group among them, by the place of its first part
  float* stats;              // [CTA][2][rows][2]: maximum and sum of a part of an item
  float* part;               // [CTA][2][rows][D]
  unsigned long long wait_ns, idle_ns;
};
cudaError_t launch_attend(AttendParams p, int max_q, int D, int num_sms, cudaStream_t stream);
cudaError_t launch_attend_many(const AttendParams& p, int D, int num_sms, cudaStream_t stream);

}  // namespace tempo
