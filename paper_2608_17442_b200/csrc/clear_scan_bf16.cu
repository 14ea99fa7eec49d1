// The sweep's kernels for one element type (a file each: they take longest to compile).
#define FESC_DBG_FILE 17   // file id in the sites a debug build reports
#include "clear_scan.cuh"

template cudaError_t scan_launch<__nv_bfloat16>(const ScanSet&, int, cudaStream_t);
