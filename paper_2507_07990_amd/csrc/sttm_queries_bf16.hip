#include "sttm_queries_kernel.h"

template void sttm::launch_queries<1>(sttm::QueryJobs&, bool, hipStream_t);  // bf16
