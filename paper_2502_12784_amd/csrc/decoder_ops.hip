// The operators around a decoder's attention (include/spark_mha.h): a source file of its own, so that it compiles beside
// spark_mha.hip.  No kernel is instantiated in both: the runtime knows a kernel by its host address.
#include "prefix_host.hpp"
#include "qk_norm_rope_host.hpp"
