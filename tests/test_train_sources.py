"""What the sources of the training-step kernels promise and no run shows (no GPU)."""
import pathlib
import re

import paper_2108_00951_gb300 as efs

CSRC = pathlib.Path(efs.__file__).parent / "csrc"


def test_what_the_launch_before_writes_is_not_read_as_constant():
    """The sorting and summing launches begin while the one before still runs: a read-only load
    (__ldg) is for memory that nothing writes meanwhile, here the caller's tokens alone."""
    text = (CSRC / "embed_grad.cu").read_text()
    loads = re.findall(r"__ldg\((.*)", text)
    assert loads and all("token" in x.split(";")[0] for x in loads)
    # the shares of layer norm's gradient likewise
    join = re.search(r"norm_join_kernel\(.*?\n}\n", (CSRC / "norm_grad.cu").read_text(), re.S).group()
    assert "griddep_wait" in join and "__ldg" not in join
