// How a forward pass is cut into workgroups.
#ifndef SLA_ATTN_PLAN_H_
#define SLA_ATTN_PLAN_H_

#include "attn.h"

namespace sla {

// Row tiles over one set of keys.  A unit is `heads` query heads of one sequence (prefix: of all sequences) that read
// the same K, V head; its rows are cut into `tiles` of 64 and its keys into `splits`.
struct AttnPart {
  int units, heads, rows, tiles, splits, blocks;
  int packed;          // rows run over the queries of several heads; else of one
  long long slot0;     // first slot of its sums
};
struct AttnPlan {
  AttnPart prefix, own;   // (prefix.blocks = 0: none)
  TileMap map;            // of `own`, where nothing is cut
  bool parts;             // sums in `part`, joined by a second launch
  long long slots;
  float *part, *stat;     // [slots][64][d], [slots][64][2]
};

AttnPlan attn_plan(const Attn& a, char* ws);
size_t attn_plan_ws(const Attn& a, const AttnPlan& p);

hipError_t attn_join(const Attn& a, const AttnPlan& plan, hipStream_t st);
hipError_t attn_forward_bf16(const Attn& a, const AttnPlan& plan, hipStream_t st);
hipError_t attn_forward_f32(const Attn& a, const AttnPlan& plan, hipStream_t st);

}  // namespace sla
#endif
