// bq4_codebook.h -- the handle behind bq4_codebook (internal to libbq): host memory only, its
// tables travel to the kernels as parameters.
#pragma once

#include "bq4_kernels.cuh"

struct bq4_codebook {
    bq4k::Tables4 tab;
};
