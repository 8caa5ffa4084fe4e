// Layout of the 8-bit key/value store.
#pragma once

#include "kernels.h"

struct pserve_kv8_s {
    int64_t places = 0;                         // tokens the store holds
    int32_t heads = 0, dim = 0;                 // key/value heads, values of a head
    int device = 0;
    int8_t *k = nullptr, *v = nullptr;          // [places][heads][dim]
    float *k_scale = nullptr, *v_scale = nullptr;   // [places][heads]
    int32_t* owner = nullptr;                   // [places] -1 between calls: the row of the running write that holds the place
    pserve::DevicePool pool;
};
