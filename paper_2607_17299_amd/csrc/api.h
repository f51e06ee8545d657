// What the sources of the C ABI share.
#pragma once

#include "../../include/war.h"
#include "kernels.h"

// Records `msg` for war_last_error and returns `code`.
war_status api_fail(war_status code, const char* msg);

struct PoolView {
  const PoolDev& dev;
  const KvGeom& geom;
  const war_model_config& cfg;
};
PoolView pool_view(const war_kv_pool* p);
