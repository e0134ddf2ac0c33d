"""Where the training loop puts its buffers.  No GPU: a model of a few numbers stands in, and the sessions are replaced."""
import torch

from paper_1704_05021_b200 import train_mlp as M


class Model:
    def __init__(self, device):
        self.device, self.shapes, self.sizes, self.layer_off = torch.device(device), [(2, 3), (3,)], [6, 3], [0, 6, 9]
        self.params = torch.zeros(9, device=device)
        self.copies = self.params.to(torch.bfloat16)


def test_buffers_lie_on_the_models_device(monkeypatch):
    """A model made elsewhere than on the first device: gradient, sum and the workers' sessions are its device's."""
    devices = []

    class Session:
        def __init__(self, *args, device=None):
            devices.append(torch.device(device))

        def push(self):
            return None

        def shard_views(self, dense):
            return dense

        def apply_call(self, *args):
            return None

    monkeypatch.setattr(M, "GradDropSession", Session)
    monkeypatch.setattr(M, "AdamWSession", lambda *args, **kw: None)
    t = M.Trainer(workers=3, model=Model("meta"))
    assert devices == [torch.device("meta")] * 3 and t.grad.device.type == t.dense.device.type == "meta"
