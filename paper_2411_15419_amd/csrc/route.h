// What the two routers share (defined in route.hip).
#pragma once

#include "luffy_common.h"

namespace luffy {

// Scratch of a routing call.
struct RouteWs {
  int32_t* hist;   // [E][k * chunks]: slots of expert e in chunk c of choice j at j * chunks + c
  int* totals;     // [E]
  int* done;       // zero before route_buckets_enqueue
};

// For chunks of as few as 16 tokens.
RouteWs carve_route(Carver& c, int T, int E, int k);

// ceil(cf*k*T/E - 1e-9), 0 without a limit.
int capacity_slots(int T, int k, int E, double cf);

// Bucket offsets, positions and tokens from topk_idx, every slot's rank among its
// chunk's slots of the same expert (in slot_pos, replaced by the position) and the
// chunks' counts in ws.hist; chunks are `tok` tokens.
void route_buckets_enqueue(const int32_t* topk_idx, int T, int E, int k, double capacity_factor, int tok,
                           int32_t* slot_pos, int32_t* perm_token, int32_t* offsets, const RouteWs& ws, hipStream_t s);

}  // namespace luffy
