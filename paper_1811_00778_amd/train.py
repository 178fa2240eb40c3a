"""Training of the plain network behind an encrypted one, and its way into the integers.

A network of network.py's layer specs is trained in the clear with PlainContext's operators -- a convolution is a product
over its placements' gathered inputs, the square activation the product's ending, the loss works on the last layer's
inputs and weights, gradients are clipped before the step (a square's slope has no bound) -- and its weights are rounded to the small
integers that hcnn_ct_scalar_mac takes (Sec. 4.3).

    python -m paper_1811_00778_amd.train [--steps S] [--batch B] [--dtype f32|f16|bf16] [--dropout P]

trains the MNIST-shaped network on made-up images, rounds it, and evaluates a few images encrypted: the decrypted scores are
the integer network's, number for number.  It also answers in the clear from weights of four bits (few_bit_scores).
"""
import numpy as np
import torch

from . import layers, network


def _inverse_table(idx, n_in):
    """For each input the positions in idx (flattened) that read it, padded with idx.size: [n_in][most readers]."""
    flat = idx.reshape(-1).astype(np.int64)
    order = np.argsort(flat, kind="stable")
    order = order[flat[order] < n_in]                          # index n_in stands for the zero of a padded border
    start = np.searchsorted(flat[order], np.arange(n_in + 1))
    most = int(np.diff(start).max(initial=0))
    table = np.full((n_in, most), flat.size, dtype=np.int64)
    for i in range(n_in):
        table[i, :start[i + 1] - start[i]] = order[start[i]:start[i + 1]]
    return table


class PlainNetwork:
    """A trainable network of network.py's specs; the last layer must be ("fc", classes).

    Weights and activations are tensors of `dtype` on the context's device; `weights` is the list of network.weight_shapes, None
    for layers without weights.  `dropout`: share of the last layer's inputs that a training step leaves out, by a mask of (seed, steps taken, image,
    input); the encrypted evaluation has none of it."""

    def __init__(self, spec, in_shape, ctx, dtype=torch.float32, seed=0, dropout=0.0):
        if spec[-1][0] != "fc":
            raise ValueError("the last layer must be fully connected: its outputs are the class scores")
        self.spec, self.in_shape, self.ctx, self.dtype = spec, in_shape, ctx, dtype
        self.seed, self.dropout, self.steps = seed, dropout, 0
        g = torch.Generator().manual_seed(seed)
        self.weights, self.tables = [], []
        prev = in_shape
        for layer, shp, ws in zip(spec, network.shapes(spec, in_shape), network.weight_shapes(spec, in_shape)):
            n_in = prev[0] * prev[1] * prev[2]
            table = None
            if layer[0] == "conv":
                idx, valid, _ = layers.conv_index_table(prev[0], prev[1], prev[2], layer[2], layer[3], layer[4], layer[5])
                idx = np.where(valid, idx, n_in)
            elif layer[0] == "pool":
                idx, _, _ = layers.pool_index_table(prev[0], prev[1], prev[2], layer[1])
            if layer[0] in ("conv", "pool"):
                table = (torch.from_numpy(idx.astype(np.int64)).to(ctx.device),
                         torch.from_numpy(_inverse_table(idx, n_in)).to(ctx.device))
            self.tables.append(table)
            if ws is None:
                self.weights.append(None)
            else:
                fan_in = int(np.prod(ws[1:]))
                self.weights.append((torch.randn(ws, generator=g) / fan_in ** 0.5).to(ctx.device, dtype))
            prev = shp

    def _gather(self, x, idx):
        """x [B][n_in] -> [B][groups][terms]; index n_in reads a zero."""
        return torch.nn.functional.pad(x, (0, 1))[:, idx]

    def _spread(self, d, inverse):
        """Gradient of _gather: every input's readers, summed in a fixed order."""
        return torch.nn.functional.pad(d.reshape(d.shape[0], -1), (0, 1))[:, inverse].sum(2)

    def _square_follows(self, i):
        return i + 1 < len(self.spec) and self.spec[i + 1][0] == "square"

    def hidden(self, x, keep=None, product=None):
        """Inputs of the last layer for images x [B][C*H*W]; `keep`: a list that takes what the backward pass needs.  product(i, rows, w, activation): (outputs, what the
        backward pass needs of them) of layer i, ctx.linear's where it is not given."""
        product = product or (lambda i, rows, w, act: self.ctx.linear(rows, w, activation=act, keep=True))
        for i, layer in enumerate(self.spec[:-1]):
            kind, saved = layer[0], None
            if kind in ("conv", "fc"):
                act = "square" if self._square_follows(i) else "none"
                w = self.weights[i].reshape(self.weights[i].shape[0], -1)
                rows = self._gather(x, self.tables[i][0]).reshape(-1, w.shape[1]) if kind == "conv" else x
                y, z = product(i, rows, w, act)
                saved = (rows, z, act)
                if kind == "conv":                              # placements x filters -> filters x placements
                    y = y.reshape(x.shape[0], -1, w.shape[0]).transpose(1, 2).reshape(x.shape[0], -1)
                x = y
            elif kind == "pool":
                x = self._gather(x, self.tables[i][0]).float().mean(2).to(self.dtype)
            elif not (i and self.spec[i - 1][0] in ("conv", "fc")):   # a square of its own
                saved = x
                x = x * x
            if keep is not None:
                keep.append(saved)
        return x

    def loss_and_gradients(self, x, labels, scale=1.0):
        """(mean loss, gradients of scale * loss for the weights, in their order)."""
        kept, grads = [], [None] * len(self.spec)
        h = self.hidden(x, kept)
        mask = (self.dropout, self.seed, self.steps % 2 ** 32)
        if self.dropout:
            h = self.ctx.dropout(h, *mask)
        loss, d, grads[-1] = self.ctx.cross_entropy_grad(h, self.weights[-1], labels, scale=scale)
        if self.dropout:
            d = self.ctx.dropout_grad(d, *mask)
        for i in range(len(self.spec) - 2, -1, -1):
            kind = self.spec[i][0]
            if kind in ("conv", "fc"):
                rows, z, act = kept[i]
                w = self.weights[i].reshape(self.weights[i].shape[0], -1)
                if kind == "conv":
                    d = d.reshape(x.shape[0], w.shape[0], -1).transpose(1, 2).reshape(-1, w.shape[0])
                first = all(layer[0] not in ("conv", "fc") for layer in self.spec[:i])
                dx, dw, _ = self.ctx.linear_grad(d, rows, w, z, activation=act, need_dx=not first)
                grads[i] = dw.reshape(self.weights[i].shape)
                if first:
                    break
                d = dx if kind == "fc" else self._spread(dx.reshape(x.shape[0], -1), self.tables[i][1])
            elif kind == "pool":
                e = self.spec[i][1]
                idx, inverse = self.tables[i]
                d = self._spread((d[:, :, None] / (e * e)).expand(-1, -1, idx.shape[1]), inverse)
            elif kept[i] is not None:
                d = 2 * d * kept[i]
        return loss, grads

    def train_step(self, x, labels, state, lr=0.05, momentum=0.9, max_norm=1.0, scale=1.0):
        """One clipped step of gradient descent with momentum (state: a dict that the caller keeps); returns (loss, norm).  Where the norm is
        not finite (binary16 gradients that overflow under their `scale`), weights and state stay as they are: the caller lowers the scale."""
        loss, grads = self.loss_and_gradients(x, labels, scale)
        self.steps += 1
        mine = [(w, g) for w, g in zip(self.weights, grads) if g is not None]
        norm = self.ctx.clip_grad_norm([g for _, g in mine], max_norm * scale)
        if "moments" not in state:
            state["master"] = [w.float() for w, _ in mine]
            state["moments"] = [torch.zeros_like(m) for m in state["master"]]
        finite = torch.isfinite(norm)                             # (decided on the device: no wait for the step)
        for (w, g), m, v in zip(mine, state["master"], state["moments"]):
            moved = (v * momentum).add_(g.float(), alpha=1.0 / scale)
            m.copy_(torch.where(finite, m.sub(moved, alpha=lr), m))
            v.copy_(torch.where(finite, moved, v))
            w.copy_(m)
        return loss, norm / scale

    def scores(self, x):
        return self.ctx.linear(self.hidden(x), self.weights[-1])

    def few_bit_weights(self):
        """Each layer's weights as a Microscaled matrix of four-bit numbers, None without weights: what few_bit_scores takes."""
        return [None if w is None else self.ctx.quantize_mx(w.reshape(w.shape[0], -1), "mx4") for w in self.weights]

    def few_bit_scores(self, x, weights, format="mx8"):
        """scores(x) with weights of four bits; the layers' inputs are rounded to `format` on their way into the products."""
        def product(i, rows, _, act):
            return self.ctx.linear_mx(self.ctx.quantize_mx(rows, format), weights[i], activation=act, dtype=self.dtype), None

        return product(len(weights) - 1, self.hidden(x, product=product), None, "none")[0]

    def integer_weights(self, bound):
        """Weights rounded to integers of magnitude at most `bound`, each layer by its own scale (int32 arrays, None without weights).  Scores
        change by a common positive factor and by rounding: the largest stays the largest where the margin allows."""
        out = []
        for w in self.weights:
            if w is None:
                out.append(None)
                continue
            v = w.float().cpu().numpy()
            out.append(np.rint(v * (bound / max(float(np.abs(v).max()), 1e-30))).astype(np.int32))
        return out


def integer_scores(spec, in_shape, weights, images):
    """The network of integer weights on integer images [B][C*H*W], exactly (Python integers where 64 bits might not do): object array."""
    x = images.astype(object)
    prev = in_shape
    for layer, shp, w in zip(spec, network.shapes(spec, in_shape), weights):
        n_in = prev[0] * prev[1] * prev[2]
        if layer[0] == "square":
            x = x * x
        elif layer[0] == "fc":
            x = x @ w.astype(object).T
        else:
            if layer[0] == "conv":
                idx, valid, _ = layers.conv_index_table(prev[0], prev[1], prev[2], layer[2], layer[3], layer[4], layer[5])
                idx = np.where(valid, idx, n_in)
            else:
                idx, _, _ = layers.pool_index_table(prev[0], prev[1], prev[2], layer[1])
            cols = np.concatenate([x, np.zeros((x.shape[0], 1), dtype=object)], 1)[:, idx]
            if layer[0] == "conv":
                x = np.transpose(cols @ w.reshape(w.shape[0], -1).astype(object).T, (0, 2, 1)).reshape(x.shape[0], -1)
            else:
                x = cols.sum(2)
        prev = shp
    return x


def encrypted_scores(spec, in_shape, weights, images, n=1024, k=11, t=5522259017729, seed=1):
    """The same scores by way of encryption: every pixel of an image becomes a ciphertext (of a constant polynomial), the network runs on
    the ciphertexts, its outputs are decrypted and read as signed numbers.  Keys and errors come from the library's samplers; n = 1024 is
    for demonstration (the paper's rings are 8192 and 16384)."""
    from . import binding
    q, p = binding.choose_moduli(n, k, t)
    ctx = binding.Context(n, q, p, t)
    s = ctx.sample_ternary(seed, 1, 1).reshape(n)
    pk, evk = ctx.keygen(s, ctx.sample_uniform(seed, 2, 1).reshape(k, n), ctx.sample_gaussian(seed, 3, 1).reshape(n),
                         ctx.sample_uniform(seed, 4, k).reshape(k, k, n), ctx.sample_gaussian(seed, 5, k))
    ctx.set_relin_key(evk)
    plan = network.Plan(spec, in_shape, weights, ctx.to_device)
    pixels, out = images.shape[1], []
    for i, image in enumerate(images):
        m = np.zeros((pixels, n), dtype=np.uint64 if ctx.wide_plaintext else np.uint32)
        m[:, 0] = image.astype(np.int64) % t
        at = 16 + 3 * i
        cts = ctx.encrypt(pk, ctx.to_device(m), ctx.sample_ternary(seed, at, pixels), ctx.sample_gaussian(seed, at + 1, pixels),
                          ctx.sample_gaussian(seed, at + 2, pixels))
        got = ctx.to_host_u32(ctx.decrypt(s, plan.run(ctx, cts)))[:, 0].astype(np.int64)
        out.append(np.where(got > t // 2, got - t, got))
    ctx.close()
    return np.stack(out)


def made_up_images(count, in_shape, classes, rng, levels=4, prototypes=None):
    """Images of `levels` grey values around a prototype for each class: (images [count][C*H*W] int, labels, prototypes)."""
    pixels = in_shape[0] * in_shape[1] * in_shape[2]
    if prototypes is None:
        prototypes = rng.integers(0, levels, size=(classes, pixels))
    labels = rng.integers(0, classes, size=count)
    noise = rng.integers(-1, 2, size=(count, pixels))
    return np.clip(prototypes[labels] + noise, 0, levels - 1).astype(np.int32), labels, prototypes


def _main(argv=None):
    import argparse
    import time

    from . import binding
    ap = argparse.ArgumentParser(prog="python -m paper_1811_00778_amd.train")
    ap.add_argument("--steps", type=int, default=150)
    ap.add_argument("--batch", type=int, default=256)
    ap.add_argument("--dtype", choices=("f32", "f16", "bf16"), default="f32")
    ap.add_argument("--lr", type=float, default=0.02)
    ap.add_argument("--bound", type=int, default=3, help="largest magnitude of the integer weights")
    ap.add_argument("--dropout", type=float, default=0.0, help="share of the last layer's inputs that a step leaves out")
    ap.add_argument("--images", type=int, default=4, help="images evaluated encrypted")
    args = ap.parse_args(argv)
    spec, in_shape, classes, levels = network.MNIST_HCNN, network.MNIST_INPUT, 10, 4
    rng = np.random.default_rng(1811)
    ctx = binding.PlainContext()
    dtype = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}[args.dtype]
    net = PlainNetwork(spec, in_shape, ctx, dtype, dropout=args.dropout)
    protos, state, scale = None, {}, 1024.0 if args.dtype == "f16" else 1.0
    t0 = time.perf_counter()
    for step in range(args.steps):
        images, labels, protos = made_up_images(args.batch, in_shape, classes, rng, levels, protos)
        x = torch.from_numpy(images).to(ctx.device, dtype) / (levels - 1)
        loss, norm = net.train_step(x, torch.from_numpy(labels).to(ctx.device), state, lr=args.lr, scale=scale)
        if args.dtype == "f16" and not np.isfinite(float(norm)):
            scale /= 2
        if step % 25 == 0 or step == args.steps - 1:
            print("step %4d  loss %.4f  gradient norm %.3f" % (step, float(loss), float(norm)), flush=True)
    print("%d steps of %d images in %.2f s" % (args.steps, args.batch, time.perf_counter() - t0))
    images, labels, _ = made_up_images(512, in_shape, classes, rng, levels, protos)
    x = torch.from_numpy(images).to(ctx.device, dtype) / (levels - 1)
    plain = net.scores(x).float().cpu().numpy()
    few = net.few_bit_scores(x, net.few_bit_weights()).float().cpu().numpy()
    weights = net.integer_weights(args.bound)
    whole = integer_scores(spec, in_shape, weights, images[:64])
    print("right answers: %.3f of 512 plain, %.3f with weights of four bits, %.3f of 64 with integer weights up to %d (largest score 2^%.1f)"
          % (float((plain.argmax(1) == labels).mean()), float((few.argmax(1) == labels).mean()), float(np.mean([int(np.argmax(r)) for r in whole] == labels[:64])), args.bound,
             np.log2(max(1, max(abs(int(v)) for r in whole for v in r)))))
    got = encrypted_scores(spec, in_shape, weights, images[:args.images])
    same = all(int(a) == int(b) for r, s in zip(got, whole) for a, b in zip(r, s))
    print("encrypted scores of %d images %s the integer network's" % (len(got), "are" if same else "DIFFER from"))
    ctx.close()
    return 0 if same else 1


if __name__ == "__main__":
    raise SystemExit(_main())
