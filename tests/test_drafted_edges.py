"""What the calls of a decode step with drafted tokens say without a GPU."""
import re
from pathlib import Path

from test_drafted_args import _cache, _tree

CSRC = Path(__file__).resolve().parent.parent / "paper_2509_22951_b200" / "csrc"


def test_the_workspace_knows_its_callers():
    """Every kernel that leaves parts in the workspace has its need in tq_attn_workspace_size."""
    size = re.search(r"int tq_attn_workspace_size\(.*?\n}", (CSRC / "tq_attn.cu").read_text(), re.S).group(0)
    users = [f for f in CSRC.glob("*.cu") if "ws.parts +" in f.read_text()]
    assert len(users) == 3
    for f in users:
        assert f.name == "tq_attn.cu" or f"{f.stem}_workspace_bytes()" in size, f.name


def test_tree_attention_counts_its_units_in_32_bits():
    """Half a billion sequences of one token and one tile: four units each over two key-value heads are more than 2^32."""
    assert _tree(_cache(), T=(1 << 29) - 1, B=1 << 30, max_pages=1) == -4
    assert _tree(_cache(), T=0, B=1 << 30, max_pages=1) == 0


def test_a_failed_query_of_a_kernel_is_not_kept():
    """The register counts that a launch checks: what is kept between calls is a count, not that there was none."""
    for name in ("tq_tree.cu", "tq_cross.cu"):
        text = (CSRC / name).read_text()
        assert "static const int regs" not in text and re.search(r"cudaFuncGetAttributes\(&a, \(const void\*\)kern\), what\)\) return rc;\s+known.store", text)
