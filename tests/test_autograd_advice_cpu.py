"""What calls say that drop a gradient: the calls that they name are there."""
import ast
import os
import re

import pytest


@pytest.fixture(scope="module")
def sg():
    import paper_2608_13757_gb300 as m
    return m


def advised(sg):
    """Every call of _not_recorded in the bindings: (its arguments as written)."""
    for module in (sg.attention, sg.cache):
        with open(module.__file__) as f:
            tree = ast.parse(f.read())
        for node in ast.walk(tree):
            if isinstance(node, ast.Call) and getattr(node.func, "id", "") == "_not_recorded":
                yield os.path.basename(module.__file__), [ast.literal_eval(a) for a in node.args], {k.arg: ast.literal_eval(k.value) for k in node.keywords}


def test_named_calls_exist(sg):
    seen = {}
    for where, args, kw in advised(sg):
        with pytest.warns(UserWarning) as w:
            sg.attention._not_recorded(*args, **kw)
        text = str(w[0].message)
        named = set(re.findall(r"sync_\w+", text))
        assert args[0] in named and all(hasattr(sg, n) for n in named), (where, text)
        assert "torch.no_grad()" in text
        seen[args[0]] = named - {args[0]}
    assert seen == {"sync_qk_norm_rope": {"sync_qk_norm_rope_backward"}, "sync_attn_forward": {"sync_attn_backward"},
                    "sync_rope": {"sync_rope_backward"}, "sync_cache_append": set(), "sync_cache_attn": set()}
