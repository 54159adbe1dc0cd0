"""The build refuses a chunk scan whose register count is not the one that its warps share out."""
import pytest

from paper_2608_23834_b200.build import check_register_split

LINE = """ptxas info    : Compiling entry function '_ZN3mkv5chunk17chunk_scan_kernelILi{d}ELi{f}EEEvNS0_6ParamsE' for 'sm_100a'
ptxas info    : Function properties for _ZN3mkv5chunk17chunk_scan_kernelILi{d}ELi{f}EEEvNS0_6ParamsE
    0 bytes stack frame, 0 bytes spill stores, 0 bytes spill loads
ptxas info    : Used {n} registers, used 1 barriers
"""


def log(n128, n256):
    other = "ptxas info    : Compiling entry function '_ZN3mkv6appendE' for 'sm_100a'\nptxas info    : Used 40 registers\n"
    return other + "".join(LINE.format(d=d, f=f, n=n) + other for d, n in ((256, n256), (128, n128)) for f in (1, 2))


def test_the_split_s_register_counts_pass():
    check_register_split(log(96, 128))


@pytest.mark.parametrize("text", [log(88, 128), log(96, 120), ""])
def test_other_counts_do_not(text):
    with pytest.raises(RuntimeError, match="chunk_scan_kernel"):
        check_register_split(text)
