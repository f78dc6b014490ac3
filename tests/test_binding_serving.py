"""The serving entry points of the binding offer no defaults that the library can only refuse."""
import inspect

import pytest

from paper_2609_24270_b200 import binding as ag


def test_the_workspace_has_to_be_given():
    p = inspect.signature(ag.attention_decode_kv4).parameters
    assert [n for n, v in p.items() if v.default is inspect.Parameter.empty][-2:] == ["workspace_ptr", "workspace_bytes"]
    pool, table = ag.KV4Pool(1 << 20, 4, 2, 64), ag.KV4Table(1 << 20, 1 << 20, 1 << 20, 2, 8)
    with pytest.raises(TypeError):
        ag.attention_decode_kv4(1 << 20, pool, table, None, 1 << 20, 1, 2)
    for kw in (dict(workspace_ptr=None, workspace_bytes=1 << 20), dict(workspace_ptr=1 << 20, workspace_bytes=0)):
        with pytest.raises(ag.AgError) as e:
            ag.attention_decode_kv4(1 << 20, pool, table, None, 1 << 20, 1, 2, **kw)
        assert e.value.status == ag.AG_ERR_ARG
