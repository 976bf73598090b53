"""The build stops where the compiler gives the prompt attention fewer registers than its roles share out."""
from paper_2509_09090_b200 import build

SOURCE = "constexpr int LAUNCH_REGS = 96, SOFTMAX_REGS = 120;"


def entry(name, regs):
    return (f"ptxas info    : Compiling entry function '{name}' for 'sm_100a'\nptxas info    : Function properties for {name}\n"
            f"    0 bytes stack frame\nptxas info    : Used {regs} registers, used 1 barriers\n")


def test_too_few_registers_are_named():
    a, b, other = "_Z3kv_prefill_tc_kernelILi64EE", "_Z3kv_prefill_tc_kernelILi128EE", "_Z3kv_decode_kernel"
    assert build.register_shortages(entry(a, 96) + entry(other, 40) + entry(b, 100), SOURCE) == []
    assert build.register_shortages(entry(a, 88) + entry(other, 128) + entry(b, 96), SOURCE) == [f"{a}: 88 registers, 96 needed"]
    assert build.register_shortages(entry(other, 128), SOURCE) == ["kv_prefill_tc_kernel: not found"]


def test_the_constant_is_read_from_the_source():
    assert build.register_shortages(entry("kv_prefill_tc_kernel", 1)) == ["kv_prefill_tc_kernel: 1 registers, 96 needed"]
