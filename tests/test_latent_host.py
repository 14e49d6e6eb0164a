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


def test_the_smaller_expanded_pool_bounds_page_ids(monkeypatch):
    """K and V pools of different sizes: ids that only the larger one has are out of range, in whichever order they come."""
    import torch

    import paper_2609_35158_b200 as pd

    counts = []

    class Recorder:
        def pd_kv_expand_latent(self, *a):
            counts.append(a[9])
            return 0

        def pd_prefill_attn_latent(self, *a):
            counts.append(a[6])
            return 0

    monkeypatch.setattr(pd, "_lib", Recorder())
    w, kv, table = torch.zeros(2, 256, 512), torch.zeros(3, 16, 576), torch.zeros(1, 3, dtype=torch.int32)
    n, ip, q, out = torch.zeros(1, dtype=torch.int32), torch.zeros(2, dtype=torch.int32), torch.zeros(1, 2, 192), torch.zeros(1, 2, 128)
    for k_count, v_count in ((7, 7), (7, 5), (4, 9)):
        k, v = torch.zeros(k_count, 2, 16, 128), torch.zeros(v_count, 2, 16, 128)
        pd.pd_kv_expand_latent(None, w, kv, table, None, n, k, v, table, stream=0)
        pd.pd_prefill_attn_latent(None, q, ip, k, v, table, kv, table, n, out, max_q_len=1, stream=0)
    assert counts == [7, 7, 5, 5, 4, 4]
