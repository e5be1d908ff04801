// The fp32 build of the 8-bit cache's combine (a second translation unit, so
// that the two compile side by side).
#define MOECA_Q8_COMBINE_F32 1
#include "q8_combine.cu"
