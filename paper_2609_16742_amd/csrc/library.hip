// Every kernel of the library as one source, so it holds one code object.
#include "kernels.hip"
#include "ops.hip"
