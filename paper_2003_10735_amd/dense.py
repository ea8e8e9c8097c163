"""A trainable 1x1 layer between a frozen front part's features and the head, trained together with the head.

The layer maps every cell of the feature map (a token) from the front's channels to the head's.  Its products run in 8-bit integers
(st_int8_linear, st_int8_linear_backward), its gradient comes from the head's full backward pass (st_partial_distill with feature_grad),
and AdamW (st_adamw_step) updates it with states of 8 or 32 bits; the head takes the library's own descent in the same call.
"""
from __future__ import annotations

import math
from dataclasses import replace

import paper_2003_10735_amd as st


class DenseFront:
    """weight [desc.c_in, c_front] float32 and bias [desc.c_in] float32 are used in place; desc describes the head behind the layer (its
    feature type and layout are chosen here: bfloat16, channels last).

    With max_norm > 0 a step whose gradients' norm is not finite leaves the layer and its state as they were, and is not counted in `steps`;
    the head, which has its own gradients, takes its step all the same.  Whether a step was taken is on the device: `step` asks for it when it
    enqueues the next one's update, behind everything else of that step, so the device has work meanwhile."""

    def __init__(self, desc: st.HeadDesc, weight, bias, lr: float = 1e-3, weight_decay: float = 0.0, max_norm: float = 1.0,
                 state_bits: int = 8):
        import torch
        self.desc = replace(desc, feat_dtype=st.ST_BF16, feat_layout=st.ST_NHWC)
        self.weight, self.bias, self.lr, self.max_norm = weight, bias, lr, max_norm
        self._steps, self._last = 0, None        # _last: recorded behind the last step, while it is not known whether it was taken
        c_out, c_front = weight.shape
        d, device = self.desc, weight.device
        cells = d.n * d.h * d.w
        self.grads = [torch.empty_like(weight), torch.empty_like(bias)]
        params = [weight, bias]
        self.tensors = st.AdamWTensors(params, self.grads, weight_decay=[weight_decay, 0.0], **st.new_adamw_state(params, state_bits))
        self.features = torch.empty((d.n, d.h, d.w, c_out), dtype=torch.bfloat16, device=device)
        self.feature_grad = torch.empty((d.n, c_out, d.h, d.w), dtype=torch.float32, device=device)
        self.loss = torch.empty(2, dtype=torch.float32, device=device)
        self.grad_norm = torch.empty(1, dtype=torch.float32, device=device)
        self._last_norm = torch.empty(1, dtype=torch.float32, pin_memory=True)
        self.workspaces = (st.new_int8_workspace(cells, c_out, c_front, device=device),
                           st.new_int8_workspace(cells, c_out, c_front, backward=True, device=device),
                           st.new_adamw_workspace(self.tensors), st.new_workspace(self.desc, device))
        self.quantized = st.st_int8_quantize(weight)

    @property
    def steps(self) -> int:
        """Steps that the layer has taken.  Waits for the last one, if it may have been left out."""
        if self._last is not None:
            self._last.synchronize()
            self._last = None
            if not math.isfinite(self._last_norm.item()):
                self._steps -= 1
        return self._steps

    @steps.setter
    def steps(self, taken: int):
        self._steps, self._last = taken, None

    def forward(self, cells):
        """cells [n*h*w, c_front], float32 or bfloat16 -> the head's features [n, h, w, c_in] bfloat16."""
        wq, scale = self.quantized
        st.st_int8_linear(cells, wq, scale, bias=self.bias, out=self.features.view(-1, self.weight.shape[0]), workspace=self.workspaces[0])
        return self.features

    def step(self, cells, labels, head_params, head_lr: float):
        """One step of the layer and of the head on one key frame (or batch).  Returns the loss before the step (on the device)."""
        import torch
        d = self.desc
        features = self.forward(cells)
        st.st_partial_distill(d, features, labels, head_params, 1, head_lr, losses=self.loss, feature_grad=self.feature_grad,
                              workspace=self.workspaces[3])
        # one frame's gradient lies channel by channel: its cells' rows are its columns, and nothing is copied
        g = self.feature_grad
        dy = g[0].view(d.c_in, d.h * d.w).t() if d.n == 1 else g.permute(0, 2, 3, 1).reshape(-1, d.c_in)
        st.st_int8_linear_backward(cells, None, dy, dw=self.grads[0], db=self.grads[1], workspace=self.workspaces[1])
        self.steps += 1
        st.st_adamw_step(self.tensors, self._steps, self.lr, max_norm=self.max_norm, grad_norm=self.grad_norm, workspace=self.workspaces[2])
        if self.max_norm > 0.0 and not torch.cuda.is_current_stream_capturing():      # (a recorded step's number is fixed)
            self._last_norm.copy_(self.grad_norm, non_blocking=True)
            self._last = torch.cuda.Event()
            self._last.record()
        st.st_int8_quantize(self.weight, *self.quantized)
        return self.loss[0]
