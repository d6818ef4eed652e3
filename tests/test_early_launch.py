"""Kernels that may become resident before the kernel ahead of them in the stream has ended (programmatic stream serialisation): what
they may touch before they wait for it.  On the CPU by reading the sources, on the GPU by a chain of them in a graph."""
import os
import re

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2607_17419_b200", "csrc")
WAIT, START = "cudaGridDependencySynchronize", "cudaTriggerProgrammaticLaunchCompletion"


def body(text, name):
    """The body of a kernel, without comments."""
    text = re.sub(r"//[^\n]*", "", text)
    at = text.index("{", re.search(r"\b%s\s*\(" % name, text).end())
    depth = 0
    for i in range(at, len(text)):
        depth += {"{": 1, "}": -1}.get(text[i], 0)
        if depth == 0:
            return text[at:i + 1]


def test_the_decode_step_lets_its_second_kernel_start_behind_its_wait():
    """decode_finish_kernel reads q and k ahead of its wait, so the kernel ahead of it must have seen their producer end before it
    lets it start (a producer that lets its own successor start early is no barrier)."""
    text = open(os.path.join(CSRC, "kata_decode.cu")).read()
    update, finish = body(text, "decode_update_kernel"), body(text, "decode_finish_kernel")
    assert finish.index("q[") < finish.index(WAIT)                # (else there is nothing to keep)
    assert 0 <= update.find(WAIT) < update.index(START)
    for name in ("q[", "k[", "v[", "S +", "Z +", "part["):
        assert update.index(WAIT) < update.index(name), name


@pytest.mark.parametrize("file", ["kata_norm_rope.cu", "kata_short_conv.cu", "kata_simt_ssm.cu", "kata_ssm_step.cu", "kata_tc_ssm.cu"])
def test_early_kernels_touch_no_memory_before_they_wait(file):
    """Every kernel of these files lets the next start before it has waited itself, so none may read or write memory before its wait:
    up to it there are only its arguments, shared memory and the tensor memory."""
    text = open(os.path.join(CSRC, file)).read()
    names = re.findall(r"__global__ void (?:__launch_bounds__\([^;{]*?\))?\s*(\w+)\s*\(", text)
    assert len(names) == text.count("__global__")
    for name in names:
        code = body(text, name)
        assert code.count("wait_for_kernels_ahead();") == 1, name
        head = re.sub(r"__shared__[^;]*;", "", code[:code.index("wait_for_kernels_ahead();")])
        for used in (r"\ba\.(q|k|v|x|out|dout|dx|positions|lengths|dt|A|D|s_init|s_final|init|local|decay|weight|bias)\b", r"\bpart\[", r"\bws\b", r"tma_load|tma_store",
                     r"sequence_length"):
            assert not re.search(used, head), (name, used)


@pytest.mark.gpu
def test_rotation_then_decode_step_in_a_graph():
    """Norm and rotation straight into the decode step, with no kernel of torch's between them, replayed again and again on changing
    inputs: to the bit what the same calls give with a synchronisation behind each."""
    import torch

    from paper_2607_17419_b200 import binding as kb

    B, H, d, steps = 4, 16, 64, 6
    gen = torch.Generator(device="cuda").manual_seed(3)
    n = lambda *s: torch.randn(*s, device="cuda", generator=gen).bfloat16()
    x, v, w = n(B, 1, 2 * H, d), n(B, H, d), 1 + 0.1 * n(d)
    S0, Z0 = torch.randn(B, H, kb.decode_n_psi(d), d, device="cuda", generator=gen), torch.rand(B, H, kb.decode_n_psi(d), device="cuda", generator=gen)
    S, Z, pos = S0.clone(), Z0.clone(), torch.zeros(1, device="cuda", dtype=torch.int64)
    qo, ko, out = (torch.empty(B, H, 1, d, device="cuda", dtype=torch.bfloat16) for _ in range(3))
    heads = x.transpose(1, 2)
    ws = kb.Workspace()

    def step():
        kb.kata_fwd_norm_rope(heads[:, :H], heads[:, H:], w, w, pos, q_out=qo, k_out=ko)
        kb.kata_decode_step(qo[:, :, 0], ko[:, :, 0], v, S, Z, out[:, :, 0], workspace=ws)

    step()                                                        # (sizes the workspace)
    torch.cuda.synchronize()
    graph, stream = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    with torch.cuda.stream(stream), torch.cuda.graph(graph, stream=stream):
        for _ in range(steps):
            step()
    for _ in range(50):
        x.copy_(n(B, 1, 2 * H, d))
        v.copy_(n(B, H, d))
        S.copy_(S0)
        Z.copy_(Z0)
        for _ in range(steps):
            kb.kata_fwd_norm_rope(heads[:, :H], heads[:, H:], w, w, pos, q_out=qo, k_out=ko)
            torch.cuda.synchronize()
            kb.kata_decode_step(qo[:, :, 0], ko[:, :, 0], v, S, Z, out[:, :, 0], workspace=ws)
            torch.cuda.synchronize()
        want, wantS, wantZ = out.clone(), S.clone(), Z.clone()
        S.copy_(S0)
        Z.copy_(Z0)
        out.zero_()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want) and torch.equal(S, wantS) and torch.equal(Z, wantZ)
