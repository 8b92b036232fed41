"""What the compiler made of the kernels of attention and rotation: what they keep of their vector registers in memory, read from the metadata of the built library."""
from paper_2411_10003_amd import binding
from test_kernel_registers import _kernels


def test_registers_in_memory():
    kernels = [k for k in _kernels(binding.LIB_PATH) if any(n in k[".name"] for n in ("attend_", "rotary_"))]
    assert len(kernels) >= 32 + 24
    in_memory = {k[".name"]: k[".private_segment_fixed_size"] for k in kernels if k[".private_segment_fixed_size"]}
    # gradients of 128 columns: of the keys' in bf16 an address of a rare branch; of the queries' in fp32 some addresses, read again in a step of 24000 clocks of products
    allowed = {"attend_dkv_kernelILi128E": 16, "attend_dq_kernelIfLi128E": 112}
    for name, size in in_memory.items():
        assert any(w in name and size <= most for w, most in allowed.items()), (name, size)
