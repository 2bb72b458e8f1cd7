// Launches of the softmax attention kernels, one function per storage type and head dimension, each an object of its own.
#pragma once
#include <hip/hip_runtime.h>

#include "ska_softmax.h"

// what: SM_FWD, SM_DQ or SM_DKV; nw: wavefronts of a workgroup, 1 or 4; args: SmArgs.  Joins the parts where there are several.
#define SKA_DECLARE_SOFTMAX(NAME) extern "C" __attribute__((visibility("hidden"))) int NAME(int what, int nw, const void *args, hipStream_t st)
SKA_DECLARE_SOFTMAX(ska_launch_softmax_f32_32);
SKA_DECLARE_SOFTMAX(ska_launch_softmax_f32_64);
SKA_DECLARE_SOFTMAX(ska_launch_softmax_f32_128);
SKA_DECLARE_SOFTMAX(ska_launch_softmax_bf16_32);
SKA_DECLARE_SOFTMAX(ska_launch_softmax_bf16_64);
SKA_DECLARE_SOFTMAX(ska_launch_softmax_bf16_128);
