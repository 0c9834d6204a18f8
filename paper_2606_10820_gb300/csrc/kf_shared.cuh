// What the kernels of shared_attention (kf_op_shared_attention) agree on: segments are query rows that read the
// same keys, those of a group's sequences its prefix (kf_shared_attention.cu, or with few rows kf_shared_rows.cu), those of a
// sequence its own keys (kf_shared_rows.cu).  They leave partial outputs, which a last kernel adds.
//
// The segments form a list that is cut into even parts.  The piece that begins a segment leaves its rows' sums at the rows' own
// places (`first`), a later one, of which a part has at most one, at the part's (`more`); the
// segment's record says where they are.
#pragma once

#include "kf_serving.cuh"

namespace kf {

struct Record { int part, pieces; };        // the part that a segment begins in, and how many have pieces of it
struct Partials {
  float* first_o;                           // [B * rows * Hq][hd], not divided by the sums
  float2* first_ml;                         // [B * rows * Hq]: reference (a raw score) and sum
  float* more_o;                            // [parts][rows of a segment][hd]
  float2* more_ml;                          // [parts][rows of a segment]
  Record* rec;                              // [segments]
  int parts, seg_rows, segments;
};
struct Sharing {
  const int32_t *groups, *shared;           // [n + 1] first sequences, [n] tokens of the prefixes
  int n;
};

// the group of sequence b (the last that begins at or before it); any lane on its own
__device__ __forceinline__ int group_of(const Sharing& s, int b) {
  int lo = 0, hi = s.n - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (__ldg(s.groups + mid) <= b) lo = mid;
    else hi = mid - 1;
  }
  return lo;
}
// a prefix's tokens (one out of range is none: its keys are then each sequence's own)
__device__ __forceinline__ int prefix_of(const Sharing& s, int g, int most) {
  const int n = __ldg(s.shared + g);
  return n >= 0 && n <= most ? n : 0;
}
// a group's sequences, in range whatever the list holds
__device__ __forceinline__ int2 members(const Sharing& s, int g, int B) {
  const int a = min(max(__ldg(s.groups + g), 0), B), b = min(max(__ldg(s.groups + g + 1), 0), B);
  return make_int2(a, max(a, b));
}
// the record of a group's tile of `seg_rows` rows under KV head hk (`before`: the rows a head that lie before the group)
__device__ __forceinline__ int prefix_record(int64_t before, int g, int tile, int seg_rows, int hk, int Hkv) {
  return (int)((before / seg_rows + g + tile) * Hkv + hk);
}
// a list of `total` places in `parts` even parts: the first `more` have one more than the others
struct Parts {
  int total, parts, each, more;
  Parts() = default;
  __device__ __forceinline__ Parts(int total_, int parts_) : total(total_), parts(parts_) {
    each = total / parts;
    more = total - each * parts;
  }
  __device__ __forceinline__ int begin(int c) const { return c < parts ? c * each + min(c, more) : total; }
  __device__ __forceinline__ int part_of(int x) const {
    const int split = more * (each + 1);
    return x < split ? x / (each + 1) : more + (x - split) / each;
  }
};

struct SharedCall {
  const void* q;
  int64_t q_seq, q_row, q_head;
  const void* pool;
  const int32_t *table, *lens;
  void* out;
  int64_t n_pages;
  Sharing sh;
  Partials pre, own;
  int* err;
  int B, rows, Hq, Hkv, G, hd, page, width;
  float scale2;
  Div by_page, by_group, by_seq, by_heads, by_rows;      // the page, the heads of a group, a sequence's rows under a KV head; Hq, rows
};

// The kernel of kf_shared_rows.cu: how many parts it has and the rows of its segments, and its launch (with the prefixes, or for
// each sequence's own keys alone, after another kernel)
struct RowsPlan { int parts, seg_rows; };
RowsPlan plan_rows(int rows_of_seq, int hd);
void launch_rows(int32_t type, const SharedCall& c, bool prefixes, cudaStream_t s);
// what paged attention says to these sizes; nullptr if they are fine
const char* paged_sizes_fault(int B, int rows, int Hq, int Hkv, int hd, int page, int width);

}  // namespace kf
