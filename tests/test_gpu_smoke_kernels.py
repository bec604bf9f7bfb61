"""smoke() runs each kernel of the attention over the paged cache: the one with the code of few items, the one without, and the join."""
import pytest

import __graft_entry__
from paper_2606_26344_b200 import gmlp

pytestmark = pytest.mark.gpu


def test_smoke_runs_the_attention_with_and_without_few_items(monkeypatch, capsys):
    plain, calls = gmlp.kv_attention, []

    def noted(*args, **kw):
        gmlp.profile_enable(True)
        try:
            O = plain(*args, **kw)
            calls.append(set(gmlp.profile_read()))
        finally:
            gmlp.profile_enable(False)
        return O

    monkeypatch.setattr(gmlp, "kv_attention", noted)
    __graft_entry__.smoke()
    assert {"kv_attention_few", "kv_join"} in calls and {"kv_attention", "kv_join"} in calls, calls
    assert len(calls) == capsys.readouterr().out.count("smoke paged attention") - 1      # one call has two requests
