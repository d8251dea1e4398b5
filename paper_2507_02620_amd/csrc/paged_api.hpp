// What the stage's own path over pages shares with the entry points of paged_api.hip.
#pragma once
#include "../../include/flowspec.h"
#include "paged.hpp"

int pool_dev(const fs_page_pool* p, PoolDev* d);                      // checks the pool's fields
int valid_rows(int dtype, int hd, const fs_kv_cache& kv);             // alignment and strides of cache rows
int valid_paged_item(const PoolDev& p, const fs_paged_item& it);      // lengths, sequence and capacity
