"""The native argument marshalling of the 8-bit cache and logits functions against the Python functions that they take over: the same
arguments reach the C entry point, however they are given.  The entry points are replaced by recorders: no GPU."""
import ctypes
import inspect
import random

import numpy as np
import pytest
import torch

import paper_2505_20776_amd as sx
from paper_2505_20776_amd import binding

sx.load_library()
NAMES = binding._marshal.QUANT_FUNCTIONS if binding._marshal is not None else ()


@pytest.fixture
def recorded():
    real = sx.load_library()
    calls, keep = {}, []

    def recorder(name):
        def note(*args):
            calls.setdefault(name, []).append(args)
            return recorder.status
        c = ctypes.CFUNCTYPE(ctypes.c_int, *[ctypes.c_void_p if t is ctypes.POINTER(sx.specext_desc) else t for t in getattr(real, "specext_" + name).argtypes])(note)
        keep.append(c)
        return c
    recorder.status = 0
    fake = type("Fake", (), {"specext_" + n: staticmethod(recorder(n)) for n in NAMES})()
    fake.specext_strerror = real.specext_strerror
    binding._lib = fake
    for n in NAMES:
        binding._marshal.bind(n, ctypes.cast(getattr(fake, "specext_" + n), ctypes.c_void_p).value)
    yield calls, recorder
    binding._lib = None
    sx.load_library()


def _argument(rng, p):
    if p.name == "desc":
        return sx.make_desc(dtype=1, n_q_heads=4, n_kv_heads=2, head_dim=64, prefix_len=9, n_tree=rng.randrange(1, 9), flags=32)
    if p.name == "check":
        return rng.choice([True, False])
    if p.name == "stream":
        return rng.choice([0, 1234, 2 ** 47 + 16])
    if p.name == "workspace_nbytes":
        return rng.choice([None, 0, 77, 2 ** 40])
    if p.name == "logit_scale":
        return rng.choice([0.0, 0.7, 1e-40, 1])
    if "stride" in p.name:
        return rng.choice([0, 128, 2 ** 40])
    if p.annotation in (int, "int"):
        return rng.choice([0, 1, -1, 7, 2 ** 31 - 1, np.int64(12), 3.0])
    tensor = torch.zeros((4, 6), dtype=rng.choice([torch.float32, torch.uint8, torch.bfloat16]))[rng.randrange(3):]
    if p.name == "workspace":
        return tensor
    return rng.choice([tensor, tensor, tensor.t(), None, 0, 4096, 2 ** 47])


def test_the_marshalling_is_there():
    assert NAMES == ("verify_attn_quant", "quant_kv_write", "quant_kv_read", "commit_tree_quant", "token_logprobs")


@pytest.mark.parametrize("name", NAMES)
def test_same_arguments_reach_the_entry_point(name, recorded):
    calls, _ = recorded
    call = getattr(sx, name)
    params = inspect.signature(call).parameters
    rng = random.Random(name)
    for _ in range(150):
        args, kwargs, by_name = [], {}, False
        for p in params.values():
            if p.default is not inspect.Parameter.empty and p.name != "stream" and rng.random() < 0.4:
                by_name = True
                continue
            by_name = by_name or rng.random() < 0.1
            if by_name:
                kwargs[p.name] = _argument(rng, p)
            else:
                args.append(_argument(rng, p))
        assert call(*args, **kwargs) == 0 and call.__wrapped__(*args, **kwargs) == 0
        native, python = calls.pop(name)
        assert native == python, (args, kwargs)


@pytest.mark.parametrize("name", NAMES)
def test_status_and_wrong_calls(name, recorded):
    calls, recorder = recorded
    call = getattr(sx, name)
    rng = random.Random(1)
    kwargs = {p.name: _argument(rng, p) for p in inspect.signature(call).parameters.values()}
    recorder.status = -2
    assert call(**{**kwargs, "check": False}) == -2
    with pytest.raises(sx.SpecextError, match="specext_" + name):
        call(**{**kwargs, "check": True})
    calls.clear()
    first = next(iter(kwargs))
    for bad in ({**kwargs, "no_such": 1}, {k: v for k, v in kwargs.items() if k != first}, {**kwargs, first: "text"}):
        with pytest.raises((TypeError, AttributeError, ctypes.ArgumentError)):
            call(**bad)
    assert not calls


def test_marshalling_of_an_older_build(tmp_path):
    """A _marshal.so without these functions is left alone: the package imports, and every call goes through ctypes."""
    import os
    import shutil
    import subprocess
    import sys
    package = os.path.dirname(os.path.abspath(binding.__file__))
    copy = tmp_path / os.path.basename(package)
    shutil.copytree(package, copy, ignore=shutil.ignore_patterns("_build*", "csrc", "_marshal.so", "__pycache__", "*.tmp"))
    (copy / "_marshal.py").write_text("FUNCTIONS = ('verify_attn',)\n")       # found where the extension would be
    (copy / "_marshal.so").write_bytes(b"")
    code = ("import importlib.machinery as m, sys; m.EXTENSION_SUFFIXES.remove('.so') if '.so' in m.EXTENSION_SUFFIXES else None\n"
            "import paper_2505_20776_amd as sx; from paper_2505_20776_amd import binding\n"
            "assert binding._marshal is None and sx.token_logprobs is binding.token_logprobs; print('fine')")
    run = subprocess.run([sys.executable, "-c", code], cwd=tmp_path, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True, timeout=250)
    assert run.returncode == 0 and "fine" in run.stdout, run.stdout[-2000:]
