"""Which memory the page cache's calls take is host arithmetic on a pointer's attributes: asked without a GPU."""

from tests.test_launch_shapes import run_program

PROGRAM = r"""
#include <cstdio>
#include <cstring>
#include "kv.cuh"
int main() {
    for (int type : {cudaMemoryTypeUnregistered, cudaMemoryTypeHost, cudaMemoryTypeDevice, cudaMemoryTypeManaged})
        for (int device : {-1, 0, 1, 3})
            for (int of : {0, 1}) {
                cudaPointerAttributes at = {};
                at.type = (cudaMemoryType)type;
                at.device = device;
                const char* what = kvdro::kv_not_usable(at, of);
                const bool fine = type == cudaMemoryTypeManaged || (type == cudaMemoryTypeDevice && device == of);
                if (fine != (what == nullptr) || (!fine && (type == cudaMemoryTypeDevice) != (std::strstr(what, "context") != nullptr))) {
                    std::printf("type %d of device %d, context of %d: %s\n", type, device, of, what ? what : "taken");
                    return 1;
                }
            }
    return 0;
}
"""


def test_memory_of_another_device_is_refused(tmp_path):
    out = run_program(tmp_path, PROGRAM)
    assert out.returncode == 0, out.stdout
