// The sweep's kernels for one element type (a file each: they take longest to compile).
#define FESC_DBG_FILE 18   // file id in the sites a debug build reports
#include "clear_scan.cuh"

template cudaError_t scan_launch<__half>(const ScanSet&, int, cudaStream_t);
