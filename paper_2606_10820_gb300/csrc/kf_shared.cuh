// What the two kernels of shared_attention (kf_op_shared_attention) agree on: the prefixes' keys
// (kf_shared_prefix.cu) and each sequence's own (kf_paged_attention.cu) leave partial outputs of every
// query row, which a last kernel adds.
//
// Either kernel takes a list of segments (rows that read the same keys) cut into even parts, one a CTA.
// The piece that begins a segment leaves its rows' sums at the rows' own places (`first`), a
// later one, of which a CTA has at most one, at the CTA's (`more`); the segment's record says where they are.
#pragma once

#include "kf_serving.cuh"

namespace kf {

constexpr int kPrefixRows = 256;            // query rows of a prefix segment
struct Record { int cta, pieces; };         // the CTA that begins a segment, and how many have pieces of it
struct Partials {
  float* first_o;                           // [B * rows * Hq][hd], not divided by the sums
  float2* first_ml;                         // [B * rows * Hq]: reference (a raw score) and sum
  float* more_o;                            // [CTAs][rows of a segment][hd]
  float2* more_ml;                          // [CTAs][rows of a segment]
  Record* rec;                              // [segments]
  int ctas, seg_rows, segments;
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
// the record of a group's pair of sub-tiles under KV head hk (`before`: the rows a head that lie before the group)
__device__ __forceinline__ int prefix_record(int64_t before, int g, int pair, int hk, int Hkv) {
  return (int)((before / kPrefixRows + g + pair) * Hkv + hk);
}

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
  Div by_page, by_group, by_seq;            // the page, the heads of a group, a sequence's rows under a KV head
};

// The kernel of each sequence's own keys (kf_paged_attention.cu): its CTAs, the rows of its segments and its records for
// these sizes, and its launch, which waits for the kernel before it only at its end
struct OwnPlan { int ctas, seg_rows, segments; };
OwnPlan plan_own(int B, int rows, int G, int Hkv, int hd, int page, int width, int64_t n_pages);
void launch_own(int32_t type, const SharedCall& c, cudaStream_t s);
// what paged attention says to these sizes; nullptr if they are fine
const char* paged_sizes_fault(int B, int rows, int Hq, int Hkv, int hd, int page, int width);

}  // namespace kf
