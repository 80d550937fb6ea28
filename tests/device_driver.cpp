// Eight threads plan at the same time, on two devices: the number of CUs of the current one, whoever asked first.
#include <cstdio>
#include <thread>
#include <vector>

#include "device.hpp"

static thread_local int current = 0;
extern "C" hipError_t hipGetDevice(int* dev) {
    *dev = current;
    return hipSuccess;
}
extern "C" hipError_t hipDeviceGetAttribute(int* value, hipDeviceAttribute_t, int dev) {
    *value = 256 + dev;
    return hipSuccess;
}

int main() {
    std::atomic<int> wrong{0};
    std::vector<std::thread> threads;
    for (int t = 0; t < 8; ++t)
        threads.emplace_back([t, &wrong] {
            current = t % 2;
            for (int i = 0; i < 1000; ++i) wrong += dlm::device_cus() != 256 + t % 2;
        });
    for (auto& t : threads) t.join();
    printf("wrong %d\n", wrong.load());
    return wrong.load() != 0;
}
