// What the attention kernels over the 4-bit cache take.
#pragma once
#include "attention_core.h"
#include "fourbit.h"

template <typename T>
struct AttentionArgs : AttentionItems<T> {
  FourBitView c;
};

// fourbit_few.hip: blocks of 16 mt rows, 4 or 8 waves that each take key tiles of their own (8: mt 1)
template <typename T>
hipError_t launch_fourbit_few(hipStream_t st, int dh, int mt, int waves, unsigned grid, const AttentionArgs<T>& a);
