// pool_view.h -- what the operators take from a pool handle.
#pragma once

#include "aqua_core.h"

namespace aqua {

struct PoolView {
    Shape shape;
    int device = 0;
    uint8_t* base = nullptr;
};

PoolView view_of(const aqua_kv_pool* pool);

}  // namespace aqua
