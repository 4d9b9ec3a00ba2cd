"""Dense layers of 8- and 16-bit operands: results and workspaces that the caller gives and the calls cannot take are refused before anything is
made for the call."""
import pytest
import torch

from paper_2008_08272_b200 import binding

M, K, F = 40, 72, 96
t = torch.bfloat16


def zeros(*size, dtype=t):
    return torch.zeros(*size, dtype=dtype, device="cuda")


def unacceptable(rows, cols):
    """In the place of a result of rows x cols: on the CPU, of a type that no call takes, of three dimensions, transposed, every second column."""
    return {"cpu": torch.zeros(rows, cols, dtype=t), "float64": zeros(rows, cols, dtype=torch.float64), "three": zeros(1, rows, cols),
            "transposed": zeros(cols, rows).T, "columns": zeros(rows, 2 * cols)[:, ::2]}


@pytest.mark.gpu
@pytest.mark.parametrize("native", [True, False])
def test_refused_before_anything_is_made(native, monkeypatch):
    X, Wg, Wu, G = zeros(M, K), zeros(F, K), zeros(F, K), zeros(M, F)
    odd = zeros(M, K + 1)[:, 1:]                       # (its copy needs a workspace)
    A, W8, sa, sw = zeros(M, K, dtype=torch.int8), zeros(F, K, dtype=torch.int8), zeros(M, dtype=torch.float32), zeros(F, dtype=torch.float32)
    calls = {"Q": (lambda **k: binding.onnx_quantize_rows(X, **k), M, K), "Y": (lambda **k: binding.onnx_gemm_int8(A, sa, W8, sw, **k), M, F),
             "dX": (lambda **k: binding.onnx_gated_backward(G, X, Wg, Wu, G, G, **k), M, K),
             "dWg": (lambda **k: binding.onnx_gated_backward(G, X, Wg, Wu, G, G, wanted=(True, False, False), **k), F, K),
             "dWu": (lambda **k: binding.onnx_gated_backward(G, X, Wg, Wu, G, G, wanted=(False, False, False), **k), F, K)}
    for name in ("H", "G", "U"):
        calls[name] = (lambda **k: binding.onnx_gated(odd, Wg, Wu, save=True, **k), M, F)
    calls["8-bit H"] = (lambda **k: binding.onnx_gated_int8(A, sa, W8, sw, W8, sw, **k), M, F)
    jobs = [(call, name.split()[-1], bad) for name, (call, rows, cols) in calls.items() for bad in unacceptable(rows, cols).values()]
    for call, bad in ((calls["Y"][0], zeros(M, K).T), (calls["dX"][0], torch.zeros(1 << 20, dtype=torch.uint8)), (calls["H"][0], zeros(1 << 12, 2)[:, 0]),
                      (calls["8-bit H"][0], torch.zeros(16))):
        jobs.append((call, "workspace", bad))
    jobs += [(calls["Q"][0], "scale", zeros(2 * M, dtype=torch.float32)[::2]), (calls["Q"][0], "scale", zeros(M))]
    if not native:
        monkeypatch.setattr(binding, "_fast_mod", binding._Declined())
    # (as many bytes as are in use now are all that there is: what a call makes is seen)
    torch.cuda.synchronize()
    torch.cuda.empty_cache()
    torch.cuda.reset_peak_memory_stats()
    before, launches = torch.cuda.memory_allocated(), binding.launch_count()
    for call, name, bad in jobs:
        with pytest.raises(TypeError):
            call(**{name: bad})
        assert torch.cuda.max_memory_allocated() == before, (name, bad.shape, bad.dtype)
    assert binding.launch_count() == launches


@pytest.mark.gpu
@pytest.mark.parametrize("native", [True, False])
def test_wanted_is_three_truth_values(native, monkeypatch):
    X, Wg, Wu, G = zeros(M, K), zeros(F, K), zeros(F, K), zeros(M, F)
    if not native:
        monkeypatch.setattr(binding, "_fast_mod", binding._Declined())
    for wanted in ((True,) * 2, (True,) * 4, (True,) * 11, ()):
        with pytest.raises(ValueError):
            binding.onnx_gated_backward(G, X, Wg, Wu, G, G, wanted=wanted)
    some = binding.onnx_gated_backward(G, X, Wg, Wu, G, G, wanted=(w for w in (1, 0, True)))
    assert [y is None for y in some] == [False, True, False]
