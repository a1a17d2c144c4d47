"""GPU: the serving calls' tests against the 64-bit definitions once more, under checks that no NaN passes (serving_checks.py): every test
of the rotation, the prompts, the drafted trees and their run together that compares with the definitions."""
import inspect

import pytest

import serving_checks
import serving_reference
import test_gpu_prompt_attend
import test_gpu_rotary
import test_gpu_serving_chain
import test_gpu_tree_attend
from test_gpu_prompt_attend import plan  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def strict(monkeypatch):
    """The strict checks in place of the others; a test that calls none of them does not belong here."""
    calls = []

    def counted(check):
        def run(*args, **kw):
            calls.append(check)
            return check(*args, **kw)
        return run

    for name in ("check_attention", "check_rotary"):
        monkeypatch.setattr(serving_reference, name, counted(getattr(serving_checks, name)))
    yield
    assert calls


for _module in (test_gpu_rotary, test_gpu_prompt_attend, test_gpu_tree_attend, test_gpu_serving_chain):
    for _name, _test in list(vars(_module).items()):
        if _name.startswith("test_") and inspect.isfunction(_test) and any(x in inspect.getsource(_test) for x in ("ref.check_", "run_case(")):
            globals()[_name.replace("test_", f"test_{_module.__name__[len('test_gpu_'):]}_", 1)] = _test
