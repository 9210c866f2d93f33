"""What the decoding loop on the cache refuses before it touches a device."""
import types

import pytest
import torch

from paper_2403_10444_b200 import cached

V, B, L, N, GAMMA = 50, 3, 7, 2, 4


def call(prompts=None, lens=None, vocabulary=V, **other):
    model = lambda n: types.SimpleNamespace(w=dict(embed=torch.zeros((n, 8)), unembed=torch.zeros((8, n))))      # noqa: E731
    i32 = lambda x: x if isinstance(x, torch.Tensor) else torch.tensor(x, dtype=torch.int32)                     # noqa: E731
    args = dict(prompts=i32([[1] * L] * B) if prompts is None else i32(prompts), prompt_lens=i32([1, 5, L] if lens is None else lens),
                u_draft=torch.zeros((N, GAMMA, B)), u_verify=torch.zeros((N, B, GAMMA + 2)))
    args.update(other)
    return cached.run(model(V), model(vocabulary), args["prompts"], args["prompt_lens"], args["u_draft"], args["u_verify"], GAMMA, algo=args.get("algo", "block_lse"))


def test_lengths_and_tokens_that_are_none_are_refused():
    row = [1] * L
    for lens in ([0, 5, L], [1, -3, L], [1, 5, L + 1], [1, 2**31 - 1, 3], [-2**31, 1, 1]):
        with pytest.raises(ValueError, match="prompt_lens"):
            call(lens=lens)
    for at, token in ((0, V), (0, -1), (4, V), (4, 2**31 - 1), (4, -2**31)):
        bad = row[:at] + [token] + row[at + 1:]
        with pytest.raises(ValueError, match="tokens"):
            call(prompts=[row, bad, row])
    with pytest.raises(ValueError, match="0 .. 29"):
        call(prompts=[row, [40] * L, row], vocabulary=30)            # (a token that one of the models does not have)


def test_shapes_that_do_not_go_together_are_refused():
    for bad in (dict(u_draft=torch.zeros((N, GAMMA + 1, B))), dict(u_verify=torch.zeros((N, B, GAMMA + 1))), dict(prompts=torch.zeros((B, L))),
                dict(lens=torch.ones((B + 1,), dtype=torch.int32)), dict(algo="greedy")):
        with pytest.raises(ValueError):
            call(**bad)
