"""Where the binding's own memory comes from, without a GPU: a call on another
stream takes it from that stream's pool.  Memory of the current stream's pool may
have been freed by a call whose kernels still run there."""
import ast
import inspect

import pytest

from paper_2606_06751_gb300 import build as B


@pytest.fixture(scope="module")
def sf():
    B.build()
    from paper_2606_06751_gb300 import stagefrontier
    return stagefrontier


class Memory:
    def __init__(self, pool):
        self.pool, self.held = pool, []

    def record_stream(self, stream):
        self.held.append(stream)


class Torch:
    """torch's streams and allocator as far as the helpers go."""

    def __init__(self):
        self.here, self.cuda = "caller", self

    def empty(self, shape, dtype, device):
        return Memory(self.here)

    def current_stream(self):
        return self.here

    def stream(self, s):
        return Within(self, s)


class Within:
    def __init__(self, torch, s):
        self.torch, self.s = torch, s

    def __enter__(self):
        self.was, self.torch.here = self.torch.here, self.s

    def __exit__(self, *_):
        self.torch.here = self.was


def test_pools(sf, monkeypatch):
    monkeypatch.setattr(sf, "torch", Torch())
    for stream, pool, held in ((None, "caller", []), ("caller", "caller", []), ("side", "side", ["caller"])):
        m = sf._new((3,), "f32", "cuda", stream)
        assert m.pool == pool and m.held == held  # read by the caller, on its own stream
        m = sf._scratch(3, "u8", "cuda", stream)
        assert m.pool == pool and m.held == []
    assert sf.torch.here == "caller"


def test_calls_on_a_stream_allocate_by_the_helpers(sf):
    tree = ast.parse(inspect.getsource(sf))
    seen = 0
    for f in ast.walk(tree):
        if not isinstance(f, ast.FunctionDef) or f.name in ("_new", "_scratch"):
            continue
        if "stream" not in [a.arg for a in f.args.args + f.args.kwonlyargs]:
            continue
        seen += 1
        for c in ast.walk(f):
            if isinstance(c, ast.Call) and isinstance(c.func, ast.Attribute):
                assert not c.func.attr.startswith(("empty", "zeros", "ones", "full")), (f.name, c.lineno)
            if isinstance(c, ast.Call) and isinstance(c.func, ast.Name):
                assert c.func.id != "rank_workspace", (f.name, c.lineno)
                if c.func.id in ("_new", "_scratch", "_empty", "_label_out"):
                    assert any(isinstance(a, ast.Name) and a.id in ("stream", "copy_stream") for a in c.args), (f.name, c.lineno)
    assert seen > 20
