// glr_operator_status after bounded waits that gave up, counted here by hand: each is reported once.  Compiled with the
// entry points themselves, linked with libglr.so for the rest.  Prints "ok" or the first violation.
#include "glr_operators.cu"

int main() {
    int* counter = gave_up_counter();
    int32_t n = -1;
    const int two = 2;
    if (!counter) { std::printf("no counter\n"); return 1; }
    if (glr_operator_status(&n) != GLR_OK || n != 0) { std::printf("at the start: %d\n", n); return 1; }
    if (cudaMemcpy(counter, &two, sizeof(two), cudaMemcpyHostToDevice) != cudaSuccess) { std::printf("copy\n"); return 1; }
    if (glr_operator_status(&n) != GLR_ETIMEOUT || n != 2) { std::printf("two events: %d\n", n); return 1; }
    if (glr_operator_status(&n) != GLR_OK || n != 0) { std::printf("once reported: %d\n", n); return 1; }
    if (glr_operator_status(nullptr) != GLR_OK) { std::printf("null\n"); return 1; }
    std::printf("ok\n");
    return 0;
}
