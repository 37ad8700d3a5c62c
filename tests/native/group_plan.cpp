// How the gated block's products are cut, for the tests: plain C++ around the header the library is built from.
#include "../../paper_2508_02322_amd/csrc/forward_plan.h"

extern "C" {
// out: small tiles or not, parts of K, M tiles, workgroups of a launch in parts
void group_plan(int bf16, int64_t groups, int64_t rows, int64_t half_columns, int64_t k_ext, int most_parts, int64_t* out) {
  const camera::GroupPlan p = camera::group_plan(bf16 != 0, groups, rows, half_columns, k_ext, most_parts);
  out[0] = p.small;
  out[1] = p.parts;
  out[2] = p.m_tiles;
  out[3] = p.blocks;
}
int64_t group_parts_bytes(int64_t product_bytes) { return camera::group_parts_bytes(product_bytes); }
}
