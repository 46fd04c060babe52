// Retrieval among the chunks in use of a cache (gca_cache_select): the decode scan over the
// landmark keys with the free slots left out (decode_scan.hpp, MASK), then one workgroup per
// retrieval row merges the scan's lists into the row's best k and writes them ascending by
// slot with their fusion weights.  The scan is bound by reading the landmarks once, the merge
// by its chain of dependent reads.
#include "cache_plan.hpp"
#include "decode_scan.hpp"

namespace gca {
namespace {

constexpr int kMergeThreads = 512;

template <int KM>
__global__ __launch_bounds__(kMergeThreads) void cache_merge_kernel(const float* __restrict__ ls,
                                                                    const int* __restrict__ lj, int64_t lists,
                                                                    int64_t pw, int K, int32_t* __restrict__ idx,
                                                                    float* __restrict__ sel, float* __restrict__ w) {
  constexpr int NW = kMergeThreads / 64;
  __shared__ float sS[NW * 32];
  __shared__ int sJ[NW * 32];
  __shared__ int sCnt[NW];
  const int lane = threadIdx.x & 63;
  const int64_t row = blockIdx.x;
  float ms;
  int mj, cnt;
  merge_lists<KM, NW>(ls, lj, row, lists, pw, K, sS, sJ, sCnt, ms, mj, cnt);
  if (threadIdx.x >= 64) return;
  const bool valid = lane < cnt;
  const int rank = rank_by_chunk(mj, cnt);
  // best first: lane 0 holds the maximum; the valid lanes sit in the lower half
  const float mx = __int_as_float(__builtin_amdgcn_readfirstlane(__float_as_int(ms)));
  const float e = valid ? expf(ms - mx) : 0.f;
  const float sum = sum32(e);
  if (lane < K) {
    const int64_t at = row * K + (valid ? rank : lane);
    idx[at] = valid ? mj : -1;
    sel[at] = valid ? ms : -INFINITY;
    if (w) w[at] = valid ? e / sum : 0.f;
  }
}

}  // namespace

hipError_t launch_cache_select(const gca_cache& c, const void* lmk_q, int32_t* idx, float* sel, float* w, void* ws,
                               hipStream_t stream) {
  const Shape s = select_shape(c);
  const hipError_t e = s.bf16 ? launch_scan<__bf16, false, true>(s, lmk_q, c.lmk, c.tokens, ws, stream)
                              : launch_scan<float, false, true>(s, lmk_q, c.lmk, c.tokens, ws, stream);
  if (e != hipSuccess) return e;
  const DecodePlan plan = decode_plan(s);
  launch_kernel("cache_merge_kernel",
                s.topk <= 8 ? cache_merge_kernel<8> : s.topk <= 16 ? cache_merge_kernel<16> : cache_merge_kernel<32>,
                dim3((unsigned)((int64_t)s.B * s.Hr)), dim3(kMergeThreads), 0, stream, decode_list_scores(s, ws),
                decode_list_chunks(s, ws), plan.lists, plan.pw, s.topk, idx, sel, w);
  return take_launch_error();
}

}  // namespace gca
