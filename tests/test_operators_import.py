"""What the package gives without torch, or with a torch build without CUDA: the declarations, the library, its argument checks."""
import os
import subprocess
import sys
import textwrap

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def _run(code):
    r = subprocess.run([sys.executable, "-c", textwrap.dedent(code)], cwd=ROOT, capture_output=True, text=True)
    assert r.returncode == 0, r.stderr
    return r.stdout


def test_the_package_is_there_without_torch():
    _run("""
        import sys
        sys.modules["torch"] = None                     # any import of it raises ImportError
        import ctypes as C
        import paper_1711_09846_b200 as pbt
        assert callable(pbt.spec_from_config) and callable(pbt.param_count) and pbt.Population
        lib = pbt.load_library()
        n = C.c_size_t(0)
        assert lib.pbt_clip_query_workspace(None, 1, 1, C.byref(n)) == 1 and lib.pbt_last_error(None)
        assert lib.pbt_adapter_forward(None, None, 0, None) == 1
        assert "AdapterProjection" in dir(pbt) and "block_norm_forward" in dir(pbt)
        try:
            pbt.AdapterProjection
        except ImportError as e:
            assert "torch" in str(e)
        else:
            raise AssertionError("the operators need torch")
        """)


def test_importing_the_package_does_not_import_torch():
    _run("""
        import sys
        import paper_1711_09846_b200 as pbt
        assert "torch" not in sys.modules
        """)


def test_the_operators_are_there_with_a_torch_without_cuda():
    _run("""
        import torch
        for name in ("_cuda_getCurrentRawStream", "_cuda_getDevice", "_cuda_cudaCachingAllocator_raw_alloc", "_cuda_cudaCachingAllocator_raw_delete"):
            delattr(torch._C, name)
        import paper_1711_09846_b200 as pbt
        from paper_1711_09846_b200 import AdapterProjection, BlockNormGrads, BlockNormOut, GradientClip, block_norm_backward, block_norm_forward
        from paper_1711_09846_b200.operators import GradientClip as same
        assert pbt.GradientClip is same and pbt.operators.GradientClip is same
        for call in (lambda: block_norm_forward(torch.zeros(1, 1, 8), next_weight=torch.ones(1, 8)), lambda: GradientClip([torch.zeros(3)]),
                     lambda: AdapterProjection(torch.zeros(4, 4), torch.zeros(1, 2, 4), torch.zeros(1, 4, 2), torch.ones(1))):
            try:
                call()
            except ValueError as e:
                assert "CUDA" in str(e)
            else:
                raise AssertionError("CPU tensors are refused")
        """)


def test_an_unknown_name_is_an_attribute_error():
    _run("""
        import paper_1711_09846_b200 as pbt
        try:
            pbt.no_such_name
        except AttributeError as e:
            assert "no_such_name" in str(e)
        else:
            raise AssertionError
        """)
