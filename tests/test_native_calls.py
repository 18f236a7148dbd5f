"""The native marshalling reads tensors as the torch that it was built with lays them out: where it is not built, or torch is another,
or a tensor is none of torch's two own classes, Python marshals."""
import importlib
import os

import numpy as np
import pytest

torch = pytest.importorskip("torch")


def test_build_without_the_headers_of_torch(tmp_path, monkeypatch, capsys):
    from paper_2304_01089_amd import build
    module = tmp_path / os.path.basename(build.CALLS)
    module.write_bytes(b"older")
    monkeypatch.setattr(build, "CALLS", str(module))
    monkeypatch.setattr(build.importlib.util, "find_spec", lambda name: None)
    assert build.build_calls() is None
    assert not module.exists() and "torch" in capsys.readouterr().err


@pytest.mark.parametrize("version", ["2.9.1", None])
def test_another_torch_than_the_one_it_was_built_with(monkeypatch, version):
    import paper_2304_01089_amd as rp
    from paper_2304_01089_amd import binding
    rp.load_library()
    calls = importlib.import_module("paper_2304_01089_amd._calls")
    assert torch.__version__.split("+")[0] == calls.torch_version
    monkeypatch.setattr(binding, "_CALLS", calls)
    monkeypatch.setattr(binding, "_CALLS_SOUGHT", False)
    if version is None:
        monkeypatch.delattr(calls, "torch_version")
    else:
        monkeypatch.setattr(calls, "torch_version", version)
    binding._set_up_calls(binding.load_library())
    assert binding._CALLS is None and binding._CALLS_SOUGHT


class Named(torch.Tensor):
    """A program's own kind of tensor."""


@pytest.mark.gpu
def test_tensors_out_of_the_ordinary():
    import paper_2304_01089_amd as rp
    from paper_2304_01089_amd import binding
    rp.load_library()
    rot = rp.rotary(64)
    x = torch.randn(5, 128, device="cuda").bfloat16()
    pos = torch.arange(5, dtype=torch.int32, device="cuda")
    want = rp.rope(rot, x, pos, 64)
    native = lambda t, p=pos, y=None: binding._CALLS.rope(t, torch.empty_like(want) if y is None else y, p, 64, 64, False, rot.freqs, 1.0, None)      # noqa: E731
    assert native(x) == 0 and native(torch.nn.Parameter(x)) == 0
    named = x.as_subclass(Named)
    assert native(named) is None
    got = torch.empty_like(want)
    rp.rope(rot, named, pos.as_subclass(Named), 64, out=got)
    assert torch.equal(got, want)
    odd = [x.to_sparse(), x.to("meta"), x[:, 0], x[None], x.t(), np.zeros((5, 128), np.float32), None, "x"]
    for t in odd:
        assert native(t) is None and native(x, t) is None and native(x, y=t if t is not None else 1) is None
