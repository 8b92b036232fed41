"""What the compiler made of the kernels of the norm and of the experts' update: no vector register in memory (in the products, whose waits count
memory operations by hand, a reload would be waited for in the place of a slice), read from the metadata of the built library."""
from paper_2411_10003_amd import binding
from test_kernel_registers import _kernels


def test_no_register_in_memory():
    kernels = [k for k in _kernels(binding.LIB_PATH) if any(n in k[".name"] for n in ("product_kernel", "few_kernel", "momentum_kernel", "start_kernel", "norm_"))]
    products = [k for k in kernels if "product_kernel" in k[".name"]]
    assert len(products) >= 24 and len(kernels) > len(products)
    # the gradients of the widest norms keep some in memory: fp32 wider than 8192, bf16 wider than that and no multiple of eight
    in_memory = {k[".name"]: k[".private_segment_fixed_size"] for k in kernels if k[".private_segment_fixed_size"]}
    assert all(any(w in n for w in ("norm_bwd_kernelIfLi1024ELi4E", "norm_bwd_kernelItLi512ELi3ELi1E", "norm_bwd_kernelItLi512ELi4ELi1E")) for n in in_memory), in_memory
