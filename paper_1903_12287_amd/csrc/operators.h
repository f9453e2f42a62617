// Launches of the operators on a caller's own tensors (include/pbg_operators.h).
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

// element types (PBG_TYPE_*)
enum { OT_F32 = 0, OT_BF16 = 1, OT_F16 = 2 };

inline int type_bytes(int type) { return type == OT_F32 ? 4 : 2; }

// bits of the device-side argument checks
enum { OPS_BAD_OFFSETS = 1, OPS_BAD_LABEL = 2 };

// ---- grouped products ---------------------------------------------------------------------------
enum { GP_FORWARD = 0, GP_DX = 1, GP_DA = 2 };

struct GroupArgs {
  const void* x;        // [n x kd]
  const void* a;        // [groups x a_group], rows of lda
  const void* dy;       // [n x md]
  void* out;            // y [n x m], dx [n x k] or da [groups x m x k]
  int64_t ldx, lda, lddy, ldo;
  int64_t a_group;      // values from a matrix to the next
  const int64_t* offsets;
  int groups;
  int64_t n;
  int k, m;             // in_dim, out_dim
  int kd, md;           // widths that the operands hold: rounded up to 16 bytes where they were packed, zeros behind
  bool a_by_row;        // a is packed with a group's matrix at place offsets[group], not at place group
  const uint32_t* bad;  // the check's verdict, read by every workgroup
  uint32_t* host_bad;   // receives it where it is not 0
};

// A slot is 2^shift rows of one group, or fewer at its end, or none.
struct GroupSlots {
  int shift;
  int64_t count;   // slots: n / 2^shift + groups
  int4* at;        // workspace: {first row, rows, group or -1, da: place of its partial sum or -1}
};

struct GroupPlan {
  bool tables;             // the tables below are written ahead of the products (else their pointers are NULL)
  GroupSlots rows;         // y, dx: a slot's rows are a tile's
  GroupSlots da;           // da: a slot's rows are summed by one workgroup
  int da_tile;             // rows and columns of a tile of da
  int64_t partial_slots;   // places of partial sums, m k floats each (0: no group is longer than a slot)
  float* partial;
  int64_t joins;           // entries of the table of groups of several sums: by group or by place, whichever are fewer
  int4* join;              // {group or -1, number of sums, place of the first}
  size_t bytes() const { return tables ? (size_t)(rows.count + da.count + joins) * 16 : 0; }
};

// what the call needs (count 0: not wanted), for workspace and launches
GroupPlan plan_group(int type, int which, int64_t n, int groups, int64_t m, int64_t k, bool want_da);
// the tables of slots, and offsets[0..groups] nondecreasing and within [0, n], else OPS_BAD_OFFSETS into *flag (nothing
// where there are no tables)
void launch_group_plan(const GroupPlan& p, const int64_t* offsets, int groups, int64_t n, uint32_t* flag,
                       hipStream_t s);
// An operand to be packed: rows of `wp` values, a multiple of 16 bytes, with zeros behind `width`.  Rows that no group
// holds are left out.
struct GroupPack {
  const void* src;
  void* dst;
  int64_t ld;           // of src; dst's rows are wp apart
  int64_t rows;         // of dst
  int matrix;           // rows of a group's matrix, one matrix a place; 0: rows of x or dy
  int width, wp;
};
// up to three of them
void launch_group_pack(int type, int count, const GroupPack* op, const int64_t* offsets, int groups, hipStream_t s);
void launch_group_product(const GroupArgs& g, int type, int which, const GroupPlan& p, hipStream_t s);

// ---- preference loss ----------------------------------------------------------------------------
struct PrefArgs {
  const void* logits;
  int64_t ld;
  const int32_t* labels;
  const int64_t* offsets;
  int pairs;
  int64_t n;
  int V;
  const float* ref;
  float beta, smoothing;
  float* loss;
  float* logp;
  float* dlogp;          // written by the loss, read by its backward
  float* stats;          // [n][2]
  double* picked;        // workspace: each row's log probability (0 where it does not count), or
  float2* parts;         // the stats of its segments, `splits` a row (0: rows are not cut)
  int splits;
  void* dlogits;
  int64_t lddl;
  uint32_t* bad;
  uint32_t* host_bad;
};

// segments of a row where they are few, else 0
int preference_splits(int64_t n, int V);
// the checks of labels and offsets, then the work
void launch_preference_loss(const PrefArgs& p, int type, hipStream_t s);
void launch_preference_backward(const PrefArgs& p, int type, hipStream_t s);

// ---- clipping -----------------------------------------------------------------------------------
constexpr int kClipBatch = 96;          // tensors a launch takes (its arguments hold their descriptors)
constexpr int kClipBlock = 8192;        // values a workgroup takes at a time

struct ClipBatch {
  const void* g[kClipBatch];
  void* o[kClipBatch];
  int64_t count[kClipBatch];
  uint32_t first[kClipBatch + 1];       // first workgroup of each tensor; first[n]: their number
  uint8_t type[kClipBatch];
  int32_t n;
  int64_t span;                         // values of a workgroup, a multiple of kClipBlock
};

// all batches: sums of squares into parts (one a workgroup, `blocks` in all), the norm into *host_norm, the scaling
void launch_clip(const ClipBatch* b, int batches, int64_t blocks, double max_norm, double* scale, double* parts,
                 double* host_norm, hipStream_t s);
