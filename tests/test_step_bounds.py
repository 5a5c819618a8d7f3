"""What the calls around new tokens ask for and refuse, on the CPU."""
import pytest

from paper_2512_01278_amd import binding as pb


@pytest.fixture(scope="module")
def lib():
    return pb.load()


def test_a_workspace_of_log_probabilities_does_for_smaller_calls(lib):
    """No call asks for more than one with as many rows, logits and alternatives, or more."""
    need = lib.pillar_logprobs_workspace_bytes
    rows = [1, 2, 3, 10, 85, 100, 128, 170, 171, 255, 256, 257, 300, 511, 512, 513, 640, 5000, 1 << 20]
    vocabs = [1, 100, 2047, 2048, 2052, 4096, 4104, 32000, 50001, 150000, 1 << 20, 1 << 30]
    for top in (0, 1, 8, 64):
        for vocab in vocabs:
            sizes = [need(r, vocab, top) for r in rows]
            assert all(s > 0 for s in sizes) and sizes == sorted(sizes), (vocab, top)
        for r in rows:
            sizes = [need(r, vocab, top) for vocab in vocabs]
            assert sizes == sorted(sizes), (r, top)
    assert need((1 << 24) - 1, 1 << 30, 64) < 1 << 20                  # rows of one part leave nothing there
