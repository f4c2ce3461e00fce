// bq4_codebook.h -- the handle behind bq4_codebook (internal to libbq): host memory only, its
// tables travel to the kernels as parameters.
#pragma once

#include "bq4_kernels.cuh"

struct bq4_codebook {
    bq4k::Tables4 tab;
    // The values times `unit` as fp16 bits, for the matrix products over a cache: unit is the smallest whole number (up to
    // 2048) that makes every value a whole number of at most 11 bits, as far as fp32 tells (the dynamic tree: 2000, a linear
    // map of n steps: n), so that the products see the values exactly; 1024 where there is none (values then round to 11 bits).
    uint16_t half[16];
    float unit;
};
