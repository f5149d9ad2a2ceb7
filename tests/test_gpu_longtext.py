"""The example that runs the paged cache's operators together.  Its attention is compared, layer by layer, with a plain
fp32 computation on the values read back: the outputs are bf16 (a relative error of at most 2^-8 each, 2^-8 / sqrt(3)
on average, so under 2^-8 of the norm), their weights off by 2^-12 at most."""
import pytest

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("args", [["--prompt", "700", "--steps", "4", "--layers", "2", "--hypotheses", "4"],
                                  ["--prompt", "64", "--steps", "2", "--layers", "1", "--hypotheses", "1", "--nodes", "1"],
                                  ["--prompt", "1285", "--steps", "3", "--layers", "2", "--hypotheses", "3", "--nodes", "40"]])
def test_example(args):
    from paper_2609_26100_gb300 import longtext
    got = longtext.main(args)
    assert got["error"] < 2.0 ** -8 + 2.0 ** -12
    if "4" == args[-1]:
        assert got["held"] < got["unshared"]
