// wq_ragged.cuh -- the sequences of a ragged batch over pages, as the attention kernels on
// pages read them on the device.
#pragma once

#include "wq_paged.h"

namespace wq {

// A sequence's first row, rows and positions; no rows where a row offset or length is out of
// range, or where the launch does not take sequences of so many rows.  len 0: a request that is not served, whose rows are zeros.
struct Seq {
  int q0, nq, len;
};
__device__ __forceinline__ Seq get_seq(const AttnPagedArgs &a, int b, bool &bad) {
  Seq s;
  s.q0 = a.cu[b];
  const int q1 = a.cu[b + 1];
  s.len = a.kv_lens[b];
  s.nq = q1 - s.q0;
  const bool none = s.len == -1;
  const bool ok = s.q0 >= 0 && q1 >= s.q0 && q1 <= a.m && s.nq <= a.max_q && (none || (s.len >= s.nq && s.len <= a.max_pages << a.shift));
  bad |= !ok;
  if (none) s.len = 0;
  if (!ok || s.nq < a.least_q || s.nq > a.most_q) s.nq = 0;
  return s;
}

}  // namespace wq
