"""Decoding in ragged chunks: room is needed for the tokens of the fullest utterance, not for the chunks' widths."""
import pytest

from test_gpu_attn_decoder_rotated import TOL, batch, make

pytestmark = pytest.mark.gpu


def test_ragged_chunks_fill_the_room_of_the_longest_utterance():
    import torch
    dec = make(dtype="f32", state_bits=32)
    room = 24
    tokens, _, states, _, frames = batch(dec, U=room)
    logp, _ = dec.forward(tokens, states, torch.full((3,), room, dtype=torch.int32, device="cuda"), frames)
    run = dec.start(states, frames, room, page=16)
    at = [0, 0, 0]

    def feed(counts, width):
        chunk = torch.zeros(3, width, dtype=torch.int64, device="cuda")
        for b, c in enumerate(counts):
            chunk[b, :c] = tokens[b, at[b]:at[b] + c]
        got = dec.extend(chunk, run, torch.tensor(counts, dtype=torch.int32, device="cuda"))
        for b, c in enumerate(counts):
            if c:
                assert (got[b, :, :c] - logp[b, :, at[b]:at[b] + c]).abs().max().item() <= TOL
            at[b] += c

    for counts in ([10, 1, 4], [0, 10, 4], [5, 0, 4], [0, 4, 10], [8, 8, 0]):  # 50 columns of chunks
        feed(counts, 10)
    assert run["filled"].tolist() == [23, 23, 22]
    with pytest.raises(ValueError, match="room"):
        dec.extend(tokens[:, :10], run, torch.tensor([0, 2, 0], dtype=torch.int32, device="cuda"))
    with pytest.raises(ValueError, match="room"):
        dec.extend(tokens[:, :2], run)
    step = dec.next(torch.stack([tokens[0, 23], tokens[1, 23], tokens[2, 22]]), run)  # (nothing that was refused left a trace)
    for b, u in enumerate((23, 23, 22)):
        assert (step[b] - logp[b, :, u]).abs().max().item() <= TOL
        at[b] += 1
    with pytest.raises(ValueError, match="room"):
        dec.next(tokens[:, 0], run)
    feed([0, 0, 1], 10)  # the shorter utterance's last one
    assert run["filled"].tolist() == [24, 24, 24]
