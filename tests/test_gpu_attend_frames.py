"""The example that runs the attention operators with the convolutions: each frame's rows against the definition."""
import numpy as np
import pytest

from paper_2207_10741_amd import binding as B, synth
from tests import attention_oracle as O, gpu_util as G

pytestmark = pytest.mark.gpu


def test_frames_attend_to_the_kept_positions_of_all_frames_so_far():
    torch = G.torch_mod()
    from examples.attend_frames import FrameAttention
    height, width, frames = 17, 23, 3
    layer = FrameAttention(height, width, frames=frames, first=1, last=1, top=2)
    oracle = O.Cache(layer.kv_heads, layer.head_dim)
    gen = torch.Generator(device="cuda:0").manual_seed(3)
    for frame in range(frames):
        x = torch.randn((1, height, width, layer.channels), generator=gen, device="cuda:0").relu_().to(torch.bfloat16)
        mask = synth.mask_objects(1, height, width, 0.5, frame)
        y, qkv, attended, selected, count = layer(x, G.mask_dev(mask))
        kept = int(mask.astype(bool).sum())
        assert int(count) == kept
        rows = G.to_f64(qkv)[:kept]
        q, k, v = rows[:, :layer.heads], rows[:, layer.heads:layer.heads + layer.kv_heads], rows[:, layer.heads + layer.kv_heads:]
        oracle.append(k, v)
        assert int(layer.length) == len(oracle)
        for i in sorted({0, 1, kept // 2, kept - 2, kept - 1}):
            position = len(oracle) - kept + i
            blocks = O.select(oracle, q[i], position, 1, 1, 2)
            assert np.array_equal(selected[i].cpu().numpy(), blocks)
            want, _, error = O.attend(oracle, q[i], position, layer.head_dim ** -0.5, True, blocks)
            off = np.abs(G.to_f64(attended[i]) - want)
            assert (off <= error + 2.0 ** -8 * (np.abs(want) + error) + 2.0 ** -133).all()
        # the last layer puts the rows back where the mask keeps them
        got = G.to_f64(y)[0]
        assert not got[mask[0] == 0].any()
        want = G.to_f64(attended)[:kept].reshape(kept, -1) @ G.to_f64(layer.w_out)[:, 0, 0].T
        rms = np.sqrt(np.mean(want ** 2))
        assert np.abs(got[mask[0] != 0] - want).max() <= 2.0 ** -8 * np.abs(want).max() + 1e-5 * rms


def test_the_example_runs(capsys):
    from examples import attend_frames
    attend_frames.main()
    assert len(capsys.readouterr().out.splitlines()) == 6
