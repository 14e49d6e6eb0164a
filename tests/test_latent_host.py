"""The latent calls as far as they can be looked at without a GPU: their sources and their bindings."""
import os
import re

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def source(name):
    return open(os.path.join(ROOT, "paper_2609_35158_b200", "csrc", name)).read()


def test_softmax_warps_give_up_as_one():
    """A bounded wait may run out in some lanes only. Where warps work together (votes, shuffles, tensor memory) no lane may leave by itself, and a
    time-out in any lane has to be latched: each way out is taken on a vote, and none is bound to the count of a loop."""
    prefill = source("pd_prefill_attn_latent.cu")
    part = prefill[prefill.index("softmax warpgroups: warpgroup t owns tile t"):prefill.index("}  // namespace")].splitlines()
    outs = [i for i, line in enumerate(part) if re.search(r"\b(break|return)\b", line) and "auto" not in line and "ok" in line]
    assert len(outs) == 2
    for i in outs:
        assert "ok = __all_sync(0xffffffffu," in part[i - 1], part[i]
    assert not any(re.search(r"for \(.*&& ok", line) for line in part)
    assert all("ok = ok && " in line or "__all_sync" in line for line in part if "mbar_wait(" in line)
    decode = source("pd_decode_attn_latent.cu")
    part = decode[decode.index("softmax: thread = (token of the tile"):decode.index("// Joins the partials")].splitlines()
    assert not any("break" in line for line in part) and all("ok = ok && " in line for line in part if "mbar_wait(" in line)
    at = next(i for i, line in enumerate(part) if "kDevTimeout" in line)
    assert "ok = __all_sync(0xffffffffu, ok);" in part[at - 1]
