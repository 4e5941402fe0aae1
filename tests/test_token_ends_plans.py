"""Workspaces of the log probabilities of a linear layer, on the host: what the largest documented sizes ask for."""
import pytest


@pytest.fixture(scope="module")
def lib():
    import os
    from paper_1805_10032_amd import binding, build
    if not os.path.exists(binding.LIB_PATH):
        build.build(verbose=False)
    return binding.load_library()


@pytest.mark.parametrize("dtype", range(3))
@pytest.mark.parametrize("rows", [65, 257, 65281, 65536, 1 << 22])
@pytest.mark.parametrize("vocab", [1 << 18, (1 << 24) - 255, 1 << 24])
def test_sums_of_a_large_vocabulary_are_kept_in_parts(lib, rows, vocab, dtype):
    """Twelve bytes for each of 2^27 sums; beside them the copies of hidden states and weights (six bytes a value, 64 M of them a plane) and a word a token."""
    got = lib.zeno_linear_logprobs_workspace_bytes(rows, vocab, 8, dtype)
    assert 0 < got <= 12 * (1 << 27) + 6 * ((64 << 20) + 8 * 65536) + 4 * 65536 + 4096
    assert got <= lib.zeno_linear_logprobs_workspace_bytes(1 << 22, vocab, 8, dtype)


def test_plans(tmp_path):
    """Which kernels the sizes of the GPU tests take, and that launches and offsets stay in their limits over the documented sizes."""
    import os
    import subprocess
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    exe = str(tmp_path / "plan_checks")
    subprocess.run(["g++", "-std=c++17", "-O2", "-fsanitize=undefined", "-fno-sanitize-recover=undefined", "-I", os.path.join(root, "include"),
                    "-I", os.path.join(root, "paper_1805_10032_amd", "csrc"), os.path.join(root, "tests", "sanitize", "plan_checks.cpp"), "-o", exe],
                   check=True, capture_output=True, text=True)
    res = subprocess.run([exe], capture_output=True, text=True, timeout=300)
    assert res.returncode == 0 and "plan checks passed" in res.stdout, res.stdout + res.stderr


@pytest.mark.parametrize("dtype", range(3))
def test_weights_of_a_few_tokens_are_packed_in_pieces(lib, dtype):
    """Copies of weights: 64 M of them a plane, in either direction.  Beside them 32 tokens' dz (four planes of 262144 values at most), their copies
    and the sums of their hidden states' gradients in eight slots."""
    rows, vocab, width = 32, 1 << 18, 1 << 13
    got = lib.zeno_linear_logprobs_backward_workspace_bytes(rows, vocab, width, dtype, 1)
    planes = 3 if dtype == 0 else 1
    assert got <= 2 * planes * (64 << 20) + 8 * rows * vocab + (8 + 8 * 4) * rows * width + 8 * width + 65536
