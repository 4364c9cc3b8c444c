// A program that changes its environment between calls, as a test that sets a knob does: what
// idle threads of earlier calls do must not read it.  (getenv in one thread while another's setenv moves the
// list reads freed memory.)  Freed blocks are written over, so that a read of one is seen.
#include <cstdio>
#include <cstdlib>
#include <cstring>
#include <string>

#include "workers.hpp"

int main(int argc, char** argv) {
    const int n = argc > 1 ? atoi(argv[1]) : 3000;
    for (int i = 0; i < n; ++i) {
        {
            sllm::TaskGroup group;
            if (group.start(8, [](uint32_t) {}) != 0) return 1;
        }  // waits for the tasks, not for what their threads do afterwards
        const std::string name = "SLLM_NOBODY_READS_" + std::to_string(i);
        setenv(name.c_str(), "1", 1);  // moves the list
        void* blocks[64];
        const size_t size = (300 + (size_t)i) * sizeof(char*);
        for (void*& b : blocks) b = std::memset(std::malloc(size), 0x5a, size);
        for (void* b : blocks) std::free(b);
    }
    std::printf("ok %u idle\n", sllm::idle_workers());
    return 0;
}
