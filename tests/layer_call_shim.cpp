// csrc/layer_call.cpp with what it asks of the HIP runtime through torch answered without a device, for tests/test_layer_call_cpu.py.
#include "../paper_2603_24517_amd/csrc/layer_call.cpp"

namespace c10::hip {
DeviceIndex current_device() { return 0; }
HIPStream getCurrentHIPStream(DeviceIndex index) { return HIPStream(HIPStream::UNCHECKED, Stream(Stream::DEFAULT, Device(DeviceType::CUDA, index))); }
hipStream_t HIPStream::stream() const { return nullptr; }
}  // namespace c10::hip
