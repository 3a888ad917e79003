#include "fd_span.cuh"
namespace fd {
size_t span_bwd_workspace_bytes(int, int, int, int, int) { return 0; }
}
