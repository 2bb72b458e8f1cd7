// Launches of the attention kernels on caches, one function per storage type, query type and head dimension, each an object of its own.
#pragma once
#include <hip/hip_runtime.h>

#include "ska_cache.h"

// nq: blocks of 16 query rows of a wavefront, 2 or 4; both: an item's workgroups take the prefix too (nq 1); args: CaArgs.  Joins the
// parts where there are several.
#define SKA_DECLARE_CACHE(NAME) extern "C" __attribute__((visibility("hidden"))) int NAME(int nq, bool both, const void *args, hipStream_t st)
#define SKA_DECLARE_CACHE_D(NAME) SKA_DECLARE_CACHE(NAME##_32); SKA_DECLARE_CACHE(NAME##_64); SKA_DECLARE_CACHE(NAME##_128)
SKA_DECLARE_CACHE_D(ska_launch_cache_f32_f32);
SKA_DECLARE_CACHE_D(ska_launch_cache_bf16_bf16);
SKA_DECLARE_CACHE_D(ska_launch_cache_e4m3_f32);
SKA_DECLARE_CACHE_D(ska_launch_cache_e4m3_bf16);
SKA_DECLARE_CACHE_D(ska_launch_cache_int8_f32);
SKA_DECLARE_CACHE_D(ska_launch_cache_int8_bf16);
