// Attention of few rows per kv head with the new tokens as a tree: the kernel of kernels_attend.cu with its masks, compiled apart so that the one without is untouched.
#define WWWS_TREE 1
#include "kernels_attend.cu"
