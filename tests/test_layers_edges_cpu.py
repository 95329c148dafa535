"""Layer operators without a GPU: refusals of the C entry points that protect memory, and the
build where torch is missing."""
import pytest

from paper_2607_11985_gb300 import binding as B


@pytest.fixture(scope="module", autouse=True)
def built():
    from paper_2607_11985_gb300 import build
    build.build()


A = 1 << 20    # an address that is never read: every call below is refused


@pytest.mark.parametrize("dtype,e", [(0, 4), (1, 2), (2, 2)])
def test_misaligned_bias_gradients_are_refused(dtype, e):
    """Outputs lie on 16-byte boundaries: the sums of a bias gradient are stored in packs."""
    def linear(gb):
        return B.lib().vqc_linear_backward(dtype, dtype, 4, 8, 8, A, 8, A, 8, A, 8, A, 2, A, A, gb, A, 1 << 30, None)

    def gated(gb, gbu):
        return B.lib().vqc_gated_backward(dtype, 4, 8, 8, A, 8, A, 8, A, A, 8, A, 3, A, A, A, gb, gbu, A, 1 << 30, None)
    for off in (e, 8):
        assert linear(A + off) == 1 and "vqc_linear_backward: misaligned" in B.vqc_last_error()
        assert gated(A + off, A) == 1 and gated(A, A + off) == 1
        assert "vqc_gated_backward: misaligned" in B.vqc_last_error()


def test_library_builds_without_torch(monkeypatch, tmp_path):
    """libvqc.so is a C library: with no torch, or one without CUDA, it is compiled and linked as
    before, and only the torch binding is left out."""
    from paper_2607_11985_gb300 import build
    real, ran = build.importlib.util.find_spec, []

    class Done:
        returncode, stdout, stderr = 0, "", ""

    def run(cmd, **_):
        ran.append(cmd)
        open(cmd[cmd.index("-o") + 1], "w").close()
        return Done

    class Spec:
        origin = str(tmp_path / "torch" / "__init__.py")       # nothing of CUDA beside it
    monkeypatch.setattr(build.subprocess, "run", run)
    monkeypatch.setattr(build, "BUILD", str(tmp_path))
    for k, found in enumerate((None, Spec)):
        monkeypatch.setattr(build.importlib.util, "find_spec", lambda name, *a: found if name == "torch" else real(name, *a))
        monkeypatch.setattr(build, "OUT", str(tmp_path / ("libvqc%d.so" % k)))
        monkeypatch.setattr(build, "OUT_LAYERS", str(tmp_path / "_layers.so"))
        ran.clear()
        assert build.build() == build.OUT
        assert len(ran) == len(build.UNITS) + 1 and not any("layers_torch" in a for cmd in ran for a in cmd)
        ran.clear()
        assert build.build() == build.OUT and not ran       # nothing has changed


def test_binding_raises_statuses():
    """The ctypes calls of the same names: sizes come back, refusals are VQCError."""
    n = B.vqc_linear_workspace_bytes(1, B.VQC_BF16, B.VQC_BF16, 64, 32, 16, 32, 32, 16, B.ACTIVATIONS["gelu"], 1)
    assert 0 < n < 1 << 20 and n % 256 == 0
    assert 0 < B.vqc_gated_workspace_bytes(1, B.VQC_F16, 64, 32, 16, 32, 32, 1) < 1 << 20
    assert 0 < B.vqc_layer_norm_workspace_bytes(64, 32) < 1 << 20
    calls = [(B.vqc_layer_norm_forward, (B.VQC_F32, 4, 8, A, 7, None, None, 1e-5, A, None, None)),
             (B.vqc_layer_norm_backward, (B.VQC_F32, 4, 8, A, 7, A, 8, None, A, A, None, None, None, 0, None)),
             (B.vqc_linear_forward, (B.VQC_F32, B.VQC_F32, 4, 8, 6, A, 7, A, 8, None, 0, None, 0, A, None, None, 0, None)),
             (B.vqc_linear_backward, (B.VQC_F32, B.VQC_F32, 4, 8, 6, A, 6, A, 7, A, 8, A, 2, A, A, A, A, 1 << 30, None)),
             (B.vqc_gated_forward, (B.VQC_F32, 4, 8, 6, A, 7, A, A, 8, None, None, 3, A, None, None, 0, None)),
             (B.vqc_gated_backward, (B.VQC_F32, 4, 8, 6, A, 6, A, 7, A, A, 8, A, 3, A, A, A, A, A, A, 1 << 30, None))]
    for call, args in calls:
        with pytest.raises(B.VQCError, match=call.__name__) as e:
            call(*args)
        assert B.STATUS[e.value.status] == "VQC_ERR_INVALID_ARG"
