"""MI355X-native MoE-offloading decode engine (arXiv 2312.17238): ctypes binding over a HIP library.

`binding` mirrors include/moe_offload.h; `engine.Stack` owns the torch-allocated memory the library
works in.  `paged` does the same for include/moe_kv.h, the paged key/value cache in 8 or 4 bits and its attention, and
`decode_loop` runs both halves of a decoder block together.  The HIP library is required: nothing here computes on the CPU.
"""
